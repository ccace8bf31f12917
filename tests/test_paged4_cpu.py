"""The paged cache in 4 bits without a GPU: refusals of the C entry points (made before anything is launched), the binding's checks,
and the plain statements that the GPU tests compare with."""
import ctypes as C

import pytest
import torch

from paper_2605_09649_b200 import binding
from util_paged4 import E4M3, LEVELS, nearest, pack, quantise, values

OK16 = 1 << 20            # an aligned address that is never followed
FIELDS = dict(k_codes=OK16, k_scales=OK16, v_codes=OK16, v_scales=OK16, k_shift=OK16, v_shift=None, n_pages=4, kv_heads=2, head_dim=64, page_size=64, reserved=0)


def cache(**kw):
    return C.byref(binding.Paged4CacheFields(**{**FIELDS, **kw}))


def append_args(cache_=None, **kw):
    a = dict(cache=cache_ or cache(), dtype=0, n=1, k=OK16, ks=128, v=OK16, vs=128, slots=OK16, status=OK16, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


def read_args(cache_=None, **kw):
    a = dict(cache=cache_ or cache(), dtype=0, n=1, slots=OK16, k=OK16, v=OK16, status=OK16, stream=None)
    assert set(kw) <= set(a)
    return list({**a, **kw}.values())


def attention_args(cache_=None, **kw):
    a = dict(cache=cache_ or cache(), dtype=0, r=1, t=1, max_new=1, hq=4, q=OK16, qs=256, cu=OK16, lens=OK16, table=OK16, width=4, scale=0.125, window=0,
             out=OK16 + (1 << 28), ws=OK16, ws_bytes=binding.paged4_workspace_bytes(4, 2, 64), status=OK16, stream=None)
    assert set(kw) <= set(a), kw
    return list({**a, **kw}.values())


def refused(fn, args, code):
    assert getattr(binding.lib(), fn)(*args) == code, binding.last_error()
    assert binding.last_error()


@pytest.mark.parametrize("kw,code", [(dict(k_codes=None), binding.E_ARG), (dict(k_scales=None), binding.E_ARG), (dict(v_codes=None), binding.E_ARG),
                                     (dict(v_scales=None), binding.E_ARG), (dict(k_codes=OK16 + 8), binding.E_ARG), (dict(v_scales=OK16 + 4), binding.E_ARG),
                                     (dict(k_shift=OK16 + 2), binding.E_ARG), (dict(v_shift=OK16 + 1), binding.E_ARG), (dict(n_pages=0), binding.E_ARG),
                                     (dict(n_pages=(1 << 24) + 1), binding.E_ARG), (dict(kv_heads=0), binding.E_ARG), (dict(kv_heads=1025), binding.E_ARG),
                                     (dict(head_dim=0), binding.E_UNSUPPORTED), (dict(head_dim=48), binding.E_UNSUPPORTED), (dict(head_dim=288), binding.E_UNSUPPORTED),
                                     (dict(page_size=32), binding.E_UNSUPPORTED), (dict(n_pages=1 << 20, kv_heads=32), binding.E_UNSUPPORTED), (dict(reserved=1), binding.E_ARG)])
def test_bad_caches_are_refused(kw, code):
    refused("trimkv_paged4_append", append_args(cache(**kw)), code)
    refused("trimkv_paged4_read", read_args(cache(**kw)), code)
    refused("trimkv_paged4_attention", attention_args(cache(**kw)), code)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(dtype=-1), dict(n=-1), dict(n=1 << 31), dict(k=None), dict(v=None), dict(slots=None), dict(k=OK16 + 8), dict(ks=127),
                                dict(vs=132), dict(ks=(1 << 31) + 8), dict(slots=OK16 + 2), dict(status=OK16 + 1)])
def test_append_refusals(kw):
    refused("trimkv_paged4_append", append_args(**kw), binding.E_ARG)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(n=-1), dict(n=1 << 31), dict(k=None), dict(v=None), dict(slots=None), dict(v=OK16 + 8), dict(slots=OK16 + 1), dict(status=OK16 + 2)])
def test_read_refusals(kw):
    refused("trimkv_paged4_read", read_args(**kw), binding.E_ARG)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(r=0), dict(r=8193), dict(t=-1), dict(t=1 << 29), dict(max_new=-1), dict(hq=1), dict(hq=3), dict(hq=258), dict(q=None), dict(q=OK16 + 8),
                                dict(qs=255), dict(qs=260), dict(cu=None), dict(lens=None), dict(table=None), dict(width=0), dict(width=16385), dict(scale=0.0), dict(scale=float("nan")),
                                dict(window=-1), dict(out=None), dict(out=OK16), dict(ws=None), dict(ws=OK16 + 16), dict(ws_bytes=100), dict(status=OK16 + 2)])
def test_attention_refusals(kw):
    refused("trimkv_paged4_attention", attention_args(**kw), binding.E_ARG)


def test_nothing_to_do_is_no_error():
    L = binding.lib()
    assert L.trimkv_paged4_append(*append_args(n=0, k=None, v=None, slots=None)) == binding.OK
    assert L.trimkv_paged4_read(*read_args(n=0, k=None, v=None, slots=None)) == binding.OK
    assert L.trimkv_paged4_attention(*attention_args(t=0, q=None, out=None)) == binding.OK
    assert binding.paged4_workspace_bytes(4, 2, 48) == binding.paged4_workspace_bytes(3, 2, 64) == binding.paged4_workspace_bytes(258, 2, 64) == 0


def test_fields_and_packed_bytes_agree():
    assert C.sizeof(binding.Paged4CacheFields) == len(binding._pack_cache4(*range(1, 12)))
    f = binding.Paged4CacheFields.from_buffer_copy(binding._pack_cache4(*range(1, 12)))
    assert [getattr(f, name) for name, _ in f._fields_] == list(range(1, 12))


def test_binding_refuses_host_tensors():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    with pytest.raises(ValueError, match="CUDA"):
        binding.Paged4Cache(u8(2, 1, 64, 16), u8(2, 1, 64, 2), u8(2, 1, 64, 16), u8(2, 1, 64, 2))


def test_plain_statement_of_the_format():
    assert E4M3[-1] == 448 and E4M3[1] == 2.0 ** -9 and E4M3[56] == 1
    assert torch.equal(E4M3, torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double())
    x = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, 7.0, 100.0], dtype=torch.float64)
    assert LEVELS[nearest(x, LEVELS)].tolist() == [0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 6.0, 6.0, 6.0]
    y = torch.zeros(1, 1, 32)
    y[0, 0, :4] = torch.tensor([6.0, -3.0, 0.5, 0.2])
    y[0, 0, 16:18] = torch.tensor([-12.0, 1.0])
    codes, scale = quantise(y, torch.zeros(1))
    assert scale.tolist() == [[[56, 64]]] and codes[0, 0, :4].tolist() == [7, 13, 1, 0] and codes[0, 0, 16:18].tolist() == [15, 1]
    back = values(pack(codes)[:, :, None], scale.to(torch.uint8)[:, :, None], torch.zeros(1))[0, 0, 0]
    assert back[:4].tolist() == [6.0, -3.0, 0.5, 0.0] and back[16:18].tolist() == [-12.0, 1.0]
    back = values(pack(codes)[:, :, None], scale.to(torch.uint8)[:, :, None], torch.tensor([-2]))[0, 0, 0]
    assert back[0] == 1.5
