"""The caller-owned paged cache without a GPU: refusals of the C entry points (made before anything is launched), the
binding's checks of tensors, and the plain statements that the GPU tests compare with."""
import ctypes as C

import pytest
import torch

from paper_2605_09649_b200 import binding
from util_paged import PAGE, Cache, attention, plan, queries, select

OK16 = 1 << 20            # an aligned address that is never followed
FIELDS = dict(k_pages=OK16, v_pages=OK16, key_bounds=OK16, n_pages=4, kv_heads=2, head_dim=64, kv_dtype=0, page_size=64, reserved=0)


def cache(**kw):
    return C.byref(binding.PagedCache(**{**FIELDS, **kw}))


def plan_args(**kw):
    a = dict(n_req=1, old=OK16, keep=OK16, new=OK16, table=OK16, width=4, free=OK16, n_pages=4, count=OK16, count_out=OK16, max_tokens=4, lens=OK16, cu=OK16,
             slots=OK16, positions=OK16, status=OK16, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


def append_args(cache_=None, **kw):
    a = dict(cache=cache_ or cache(), n=1, k=OK16, ks=128, v=OK16, vs=128, slots=OK16, status=OK16, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


def attention_args(cache_=None, sparse=False, **kw):
    need = binding.paged_workspace_bytes(4, 2, 64)
    a = dict(cache=cache_ or cache(), r=1, t=1, max_new=1, hq=4, q=OK16, qs=256, cu=OK16, lens=OK16, table=OK16, width=4, scale=0.125)
    a.update(dict(top=3, sink=1, recent=1, selected=OK16) if sparse else dict(window=0))
    a.update(out=OK16 + (1 << 28), ws=OK16, ws_bytes=need, status=OK16, stream=None)
    if sparse:
        del a["max_new"]
    assert set(kw) <= set(a), kw
    return list({**a, **kw}.values())


def refused(fn, args, code):
    assert getattr(binding.lib(), fn)(*args) == code, binding.last_error()
    assert binding.last_error()


BAD_CACHES = [(dict(k_pages=None), binding.E_ARG), (dict(v_pages=None), binding.E_ARG), (dict(k_pages=OK16 + 8), binding.E_ARG),
              (dict(key_bounds=OK16 + 2), binding.E_ARG), (dict(n_pages=0), binding.E_ARG), (dict(n_pages=(1 << 24) + 1), binding.E_ARG),
              (dict(kv_heads=0), binding.E_ARG), (dict(kv_heads=1025), binding.E_ARG), (dict(head_dim=0), binding.E_UNSUPPORTED),
              (dict(head_dim=12), binding.E_UNSUPPORTED), (dict(head_dim=264), binding.E_UNSUPPORTED), (dict(kv_dtype=2), binding.E_ARG),
              (dict(n_pages=1 << 20, kv_heads=32), binding.E_UNSUPPORTED), (dict(page_size=32), binding.E_UNSUPPORTED), (dict(reserved=1), binding.E_ARG)]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_bad_caches_are_refused(kw, code):
    refused("trimkv_paged_append", append_args(cache(**kw)), code)
    refused("trimkv_paged_attention", attention_args(cache(**kw)), code)
    refused("trimkv_paged_sparse_attention", attention_args(cache(**kw), sparse=True), code)


@pytest.mark.parametrize("kw", [dict(n_req=0), dict(n_req=8193), dict(width=0), dict(width=16385), dict(n_pages=0), dict(n_pages=(1 << 24) + 1),
                                dict(max_tokens=-1), dict(max_tokens=(1 << 30) + 1), dict(old=None), dict(new=None), dict(table=None), dict(free=None),
                                dict(count=None), dict(count_out=None), dict(lens=None), dict(cu=None), dict(slots=None), dict(slots=OK16 + 4),
                                dict(positions=OK16 + 8), dict(old=OK16 + 2), dict(status=OK16 + 1)])
def test_plan_refusals(kw):
    refused("trimkv_paged_plan", plan_args(**kw), binding.E_ARG)


@pytest.mark.parametrize("kw", [dict(n=-1), dict(n=1 << 31), dict(k=None), dict(v=None), dict(slots=None), dict(k=OK16 + 4), dict(v=OK16 + 8), dict(ks=127), dict(vs=120),
                                dict(ks=132), dict(slots=OK16 + 2), dict(ks=(1 << 31) + 8)])
def test_append_refusals(kw):
    refused("trimkv_paged_append", append_args(**kw), binding.E_ARG)


COMMON = [dict(r=0), dict(r=8193), dict(t=-1), dict(t=1 << 29), dict(hq=1), dict(hq=3), dict(hq=258), dict(q=None), dict(q=OK16 + 2), dict(qs=255), dict(qs=260),
          dict(cu=None), dict(lens=None), dict(table=None), dict(width=0), dict(width=16385), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
          dict(scale=float("inf")), dict(out=None), dict(out=OK16 + 4), dict(out=OK16), dict(t=3, out=OK16 + 2 * 512 + 256), dict(q=OK16 + (1 << 28) + 256), dict(ws=None), dict(ws=OK16 + 16), dict(ws_bytes=0), dict(cu=OK16 + 1), dict(status=OK16 + 2)]


@pytest.mark.parametrize("kw", COMMON + [dict(window=-1), dict(window=(1 << 30) + 1), dict(max_new=-1)])
def test_attention_refusals(kw):
    refused("trimkv_paged_attention", attention_args(**kw), binding.E_ARG)


@pytest.mark.parametrize("kw", COMMON + [dict(sink=-1), dict(recent=0), dict(top=1), dict(top=0), dict(top=16385), dict(sink=2 ** 31 - 1), dict(selected=None)])
def test_sparse_attention_refusals(kw):
    refused("trimkv_paged_sparse_attention", attention_args(sparse=True, **kw), binding.E_ARG)


def test_sparse_attention_needs_bounds_and_a_table_that_fits():
    refused("trimkv_paged_sparse_attention", attention_args(cache(key_bounds=None), sparse=True), binding.E_ARG)
    need = binding.paged_workspace_bytes(128, 1, 256)
    refused("trimkv_paged_sparse_attention", attention_args(cache(kv_heads=1, head_dim=256, kv_dtype=1), sparse=True, hq=128, qs=128 * 256, ws_bytes=need), binding.E_UNSUPPORTED)


def test_calls_without_tokens_launch_nothing():
    before = binding.kernel_launches()
    L = binding.lib()
    assert L.trimkv_paged_append(*append_args(n=0, k=None, v=None, slots=None)) == binding.OK
    assert L.trimkv_paged_attention(*attention_args(t=0, q=None, out=None)) == binding.OK
    assert L.trimkv_paged_sparse_attention(*attention_args(sparse=True, t=0, q=None, out=None, selected=None)) == binding.OK
    assert binding.kernel_launches() == before


def test_workspace_bytes():
    assert binding.paged_workspace_bytes(32, 8, 128) > 0
    for bad in ((32, 0, 128), (33, 8, 128), (4, 8, 128), (32, 8, 12), (32, 8, 264), (129, 1, 64)):
        assert binding.paged_workspace_bytes(*bad) == 0


def test_workspace_bytes_hold_what_a_head_size_can_use():
    """Of each kernel: a note of 16 bytes per worker and two partial results (m, l, O in fp32) per row of its workers' units: 148 x 2 x 64
    rows everywhere, 148 x 256 more where the tensor-core kernel takes the head size (up to 128)."""
    part = lambda rows, d: 148 * 4 * 16 + 2 * rows * (d + 2) * 4
    for d in (8, 64, 96, 128):
        assert 0 <= binding.paged_workspace_bytes(16, 4, d) - part(148 * 128, d) - part(148 * 256, d) < 512, d
    for d in (136, 192, 256):
        assert 0 <= binding.paged_workspace_bytes(16, 4, d) - part(148 * 128, d) < 256, d


def test_binding_refuses_wrong_tensors():
    kp = torch.zeros(2, 2, PAGE, 64)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.paged_attention(kp, kp, torch.zeros(1, 4, 64), torch.zeros(2, dtype=torch.int32), i, i[None], 1)      # CPU tensors
    with pytest.raises(ValueError):
        binding.paged_append(kp, kp, kp[:1, :, 0], kp[:1, :, 0], i)
    with pytest.raises(ValueError):
        binding.paged_plan(i, i, i, i[None], i, i, i, i, i, i)
    dev = -1                                                               # what get_device says of a CPU tensor
    for bad in (torch.zeros(3, 4, 64)[:, :, ::2], torch.zeros(3, 8, 32)[:, ::2], torch.zeros(3, 4, 32, dtype=torch.float64), torch.zeros(3, 5, 32), torch.zeros(3, 128)):
        with pytest.raises(ValueError):
            binding._rows(dev, "q", bad, torch.float32, 4, 32)
    assert binding._rows(dev, "q", torch.zeros(3, 6, 32)[:, :4], torch.float32, 4, 32)[1] == 192       # strided tokens
    for bad in (torch.zeros(3, 4)[:, ::2], torch.zeros(4), torch.zeros(3, 4, dtype=torch.int64), torch.zeros(2, 4)):
        with pytest.raises(ValueError):
            binding._on(dev, "x", bad, torch.float32, (3, 4))


# ---- the plain statements themselves

def test_binding_refuses_numbers_that_do_not_fit_32_bits():
    z = torch.zeros(1)
    for kw in (dict(window=(1 << 32) + 5), dict(max_new=1 << 31)):
        with pytest.raises(ValueError, match=next(iter(kw))):
            binding.paged_attention(z, z, z, z, z, z, **kw)
    for kw in (dict(top_pages=(1 << 32) + 3), dict(top_pages=3, sink_pages=1 << 32), dict(top_pages=3, recent_pages=(1 << 32) + 1)):
        with pytest.raises(ValueError, match=list(kw)[-1]):
            binding.paged_sparse_attention(z, z, z, z, z, z, z, **kw)


def test_plain_plan_by_hand():
    got = plan([70, 130, 0], [70, 60, 0], [129, 61, 2], [[9, 8, 0], [7, 6, 5], [0, 0, 0]], [1, 2, 0, 0, 0, 0], 2, 64)
    # request 1 gives back 6 and 5; request 0 pops 5, request 2 pops 6
    assert got[0] == [[9, 8, 5], [7, 6, 5], [6, 0, 0]]
    assert got[1] == [1, 2, 6, 5, 0, 0] and got[2] == 2 and got[3] == [129, 61, 2]
    assert got[4] == [0, 59, 60, 62]
    assert got[5][0] == 8 * 64 + 6 and got[5][58:62] == [5 * 64, 7 * 64 + 60, 6 * 64, 6 * 64 + 1] and got[5][62:] == [-1, -1]


def test_plain_attention_equals_a_dense_softmax_and_selection_of_all_pages():
    c = Cache([150, 64], 2, 16, torch.float32, "cpu", 3)
    q, cu = queries([4, 1], 4, 16, torch.float32, "cpu", 3)
    out, bound, _ = attention(c.k, c.v, q, cu, [150, 64], c.table, 0.25)
    k = torch.cat([c.k[p] for p in c.table[0].tolist()], 1)[:, :150].double()
    v = torch.cat([c.v[p] for p in c.table[0].tolist()], 1)[:, :150].double()
    for j in range(4):
        for hq in range(4):
            n = 147 + j
            want = torch.softmax(k[hq // 2, :n] @ q[j, hq].double() * 0.25, 0) @ v[hq // 2, :n]
            assert torch.allclose(out[j, hq], want, atol=1e-12)
    same, _, sel = attention(c.k, c.v, q, cu, [150, 64], c.table, 0.25, 0, c.bounds, 3, 0, 1)
    assert torch.equal(same, out) and sel[0, 0].tolist() == [0, 1, 2] and sel[4, 1].tolist() == [0, -1, -1]
    assert (bound > 0).all()


def test_plain_selection_bounds_every_key():
    gen = torch.Generator().manual_seed(1)
    k, q = torch.randn(9, PAGE, 8, generator=gen).double(), torch.randn(3, 8, generator=gen).double()
    b = torch.stack((k.amin(1), k.amax(1)), 1)
    u = torch.maximum(q[:, None] * b[None, :, 0], q[:, None] * b[None, :, 1]).sum(-1)
    assert (u >= (q @ k.flatten(0, 1).T).unflatten(1, (9, PAGE)).amax(-1)).all()
    best = u.amax(0)[1:7].argmax().item() + 1
    assert select(q, b, 9, 4, 1, 2) == sorted([0, best, 7, 8])
