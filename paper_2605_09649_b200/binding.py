"""Thin ctypes binding of the trimkv C ABI (include/trimkv.h).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.  torch tensors
supply device memory and the current stream.  There is no CPU fallback: if the shared library has not
been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtrimkv.so")

OK, E_ARG, E_STATE, E_NOMEM, E_CUDA, E_NONFINITE, E_TIMEOUT, E_UNSUPPORTED = range(8)
STATUS_NAMES = ["OK", "E_ARG", "E_STATE", "E_NOMEM", "E_CUDA", "E_NONFINITE", "E_TIMEOUT", "E_UNSUPPORTED"]
DTYPE_BF16, DTYPE_F32 = 0, 1
TEST_DISTRUST_SAMPLE, TEST_ATTENTION_NO_COPY, TEST_UNION_OF_PAGES = 1, 2, 4     # testing aids, see trimkv_set_test_hooks

EXPORTS = [
    "trimkv_default_config", "trimkv_create", "trimkv_create_ex", "trimkv_destroy", "trimkv_reset", "trimkv_set_gate",
    "trimkv_set_shared_projection", "trimkv_gate", "trimkv_append", "trimkv_score_and_evict", "trimkv_decode_attention",
    "trimkv_prefill_attention", "trimkv_decode_step_all", "trimkv_decode_step_all_host", "trimkv_get_lengths", "trimkv_get_kept", "trimkv_get_pool", "trimkv_get_select_stats",
    "trimkv_sync_status", "trimkv_set_overlap", "trimkv_set_horizon", "trimkv_profile", "trimkv_profile_read", "trimkv_last_error", "trimkv_kernel_launches", "trimkv_select_workspace_bytes",
    "trimkv_select_topk", "trimkv_select_topk_static", "trimkv_set_test_hooks",
    "trimkv_step_stream", "trimkv_check_invariants", "trimkv_import_pool", "trimkv_import_finish", "trimkv_shard_sample_cap", "trimkv_shard_sample", "trimkv_shard_bracket", "trimkv_shard_filter", "trimkv_shard_candidates",
    "trimkv_shard_resolve", "trimkv_shard_hist", "trimkv_shard_digit", "trimkv_shard_mark", "trimkv_shard_compact",
    "trimkv_paged_plan", "trimkv_paged_append", "trimkv_paged_workspace_bytes", "trimkv_paged_attention",
    "trimkv_paged_sparse_attention",
    "trimkv_paged4_append", "trimkv_paged4_read", "trimkv_paged4_workspace_bytes", "trimkv_paged4_attention",
    "trimkv_paged_share", "trimkv_paged_compact", "trimkv_paged_move",
]


class TrimkvError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"trimkv {STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else status}: {message}")
        self.status = status


class Config(C.Structure):
    _fields_ = [
        ("budget_entries", C.c_int64), ("layers", C.c_int32), ("kv_heads", C.c_int32), ("q_heads", C.c_int32),
        ("head_dim", C.c_int32), ("hidden", C.c_int32), ("max_batch", C.c_int32), ("page_size", C.c_int32),
        ("gate_hidden", C.c_int32), ("gate_embed", C.c_int32), ("horizon", C.c_int32), ("kv_dtype", C.c_int32),
        ("max_chunk", C.c_int32), ("reserved", C.c_int32), ("max_pool_pages", C.c_int64),
        ("retention_bias", C.c_int32), ("per_pool_budget", C.c_int32),
        ("shard_total_layers", C.c_int32), ("shard_layer0", C.c_int32),
    ]


class PagedCache(C.Structure):
    """trimkv_paged_cache: the page arrays of a caller-owned cache."""
    _fields_ = [
        ("k_pages", C.c_void_p), ("v_pages", C.c_void_p), ("key_bounds", C.c_void_p), ("n_pages", C.c_int32),
        ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("kv_dtype", C.c_int32), ("page_size", C.c_int32),
        ("reserved", C.c_int32),
    ]


class Paged4CacheFields(C.Structure):
    """trimkv_paged4_cache: the arrays of a caller-owned cache in 4 bits."""
    _fields_ = [
        ("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p),
        ("k_shift", C.c_void_p), ("v_shift", C.c_void_p), ("n_pages", C.c_int32), ("kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("page_size", C.c_int32), ("reserved", C.c_int32),
    ]


class PagedRows(C.Structure):
    """trimkv_paged_rows: an array of pages whose rows are moved."""
    _fields_ = [
        ("pages", C.c_void_p), ("key_bounds", C.c_void_p), ("heads", C.c_int32), ("row_bytes", C.c_int32),
        ("dtype", C.c_int32), ("reserved", C.c_int32),
    ]


_lib = None


def lib() -> C.CDLL:
    """Load the shared library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2605_09649_b200.build` "
                           "(there is no fallback path)")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int, C.c_int64, C.c_float
    L.trimkv_default_config.argtypes = [C.POINTER(Config), i64, i32, i32, i32]
    L.trimkv_default_config.restype = None
    L.trimkv_create.argtypes = [i64, i32, i32, i32]
    L.trimkv_create.restype = vp
    L.trimkv_create_ex.argtypes = [C.POINTER(Config), C.POINTER(vp)]
    L.trimkv_destroy.argtypes = [vp]
    L.trimkv_destroy.restype = None
    L.trimkv_reset.argtypes = [vp]
    L.trimkv_set_gate.argtypes = [vp, i32, vp, vp, vp, vp]
    L.trimkv_set_shared_projection.argtypes = [vp, vp, f32]
    L.trimkv_gate.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp]
    L.trimkv_append.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp]
    L.trimkv_score_and_evict.argtypes = [vp, vp]
    L.trimkv_decode_attention.argtypes = [vp, i32, vp, vp, vp]
    L.trimkv_prefill_attention.argtypes = [vp, i32, i32, vp, vp, vp]
    L.trimkv_prefill_attention.restype = i32
    L.trimkv_decode_step_all.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    L.trimkv_decode_step_all_host.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
    L.trimkv_decode_step_all_host.restype = i32
    L.trimkv_get_lengths.argtypes = [vp, vp]
    L.trimkv_get_kept.argtypes = [vp, i32, i32, i32, vp, i32, C.POINTER(i32)]
    L.trimkv_get_pool.argtypes = [vp, i32, i32, i32, i32, C.POINTER(i32), vp, vp, vp, vp, vp]
    L.trimkv_get_select_stats.argtypes = [vp, vp]
    L.trimkv_sync_status.argtypes = [vp]
    L.trimkv_profile.argtypes = [vp, i32]
    L.trimkv_set_overlap.argtypes = [vp, i32]
    L.trimkv_set_test_hooks.argtypes = [vp, i32]
    L.trimkv_step_stream.argtypes = [vp]
    L.trimkv_check_invariants.argtypes = [vp]
    L.trimkv_check_invariants.restype = i32
    L.trimkv_import_pool.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp]
    L.trimkv_import_pool.restype = i32
    L.trimkv_import_finish.argtypes = [vp, i64]
    L.trimkv_import_finish.restype = i32
    L.trimkv_step_stream.restype = vp
    L.trimkv_shard_sample_cap.argtypes = []
    L.trimkv_shard_sample.argtypes = [vp, i64, i64, vp, vp, vp]
    L.trimkv_shard_bracket.argtypes = [vp, i32, vp, vp, i64, i64, vp]
    L.trimkv_shard_filter.argtypes = [vp, vp, vp, vp]
    L.trimkv_shard_candidates.argtypes = [vp, i64, vp, vp]
    L.trimkv_shard_resolve.argtypes = [vp, i32, i32, i64, vp, vp, vp, i64, vp, vp]
    L.trimkv_shard_hist.argtypes = [vp, vp, i32, vp, vp]
    L.trimkv_shard_digit.argtypes = [vp, vp, vp, vp, i32, vp]
    L.trimkv_shard_mark.argtypes = [vp, vp, vp]
    L.trimkv_shard_compact.argtypes = [vp, vp, vp]
    L.trimkv_set_horizon.argtypes = [vp, i32, vp]
    L.trimkv_profile_read.argtypes = [vp, vp, vp]
    L.trimkv_last_error.argtypes = []
    L.trimkv_last_error.restype = C.c_char_p
    L.trimkv_kernel_launches.argtypes = []
    L.trimkv_kernel_launches.restype = i64
    L.trimkv_select_workspace_bytes.argtypes = [i64]
    L.trimkv_select_workspace_bytes.restype = C.c_size_t
    L.trimkv_select_topk.argtypes = [vp, i64, i64, vp, vp, C.c_size_t, vp, vp]
    L.trimkv_select_topk_static.argtypes = [vp, i64, i64, vp, vp, vp]
    pc, sz = C.c_void_p, C.c_size_t          # pc: trimkv_paged_cache*, byref(PagedCache(...)) or its bytes
    L.trimkv_paged_plan.argtypes = [i32, vp, vp, vp, vp, i32, vp, i32, vp, vp, i64, vp, vp, vp, vp, vp, vp]
    L.trimkv_paged_append.argtypes = [pc, i64, vp, i64, vp, i64, vp, vp, vp]
    L.trimkv_paged_workspace_bytes.argtypes = [i32, i32, i32]
    L.trimkv_paged_workspace_bytes.restype = sz
    L.trimkv_paged_attention.argtypes = [pc, i32, i64, i32, i32, vp, i64, vp, vp, vp, i32, f32, i32, vp, vp, sz, vp, vp]
    L.trimkv_paged4_append.argtypes = [pc, i32, i64, vp, i64, vp, i64, vp, vp, vp]      # pc: trimkv_paged4_cache* likewise
    L.trimkv_paged4_read.argtypes = [pc, i32, i64, vp, vp, vp, vp, vp]
    L.trimkv_paged4_workspace_bytes.argtypes = [i32, i32, i32]
    L.trimkv_paged4_workspace_bytes.restype = sz
    L.trimkv_paged4_attention.argtypes = [pc, i32, i32, i64, i32, i32, vp, i64, vp, vp, vp, i32, f32, i32, vp, vp, sz, vp, vp]
    L.trimkv_paged_share.argtypes = [i32, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, i64, vp, vp, vp, vp, i64, vp, vp, vp, vp, vp]
    L.trimkv_paged_compact.argtypes = [i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, vp, i64, vp, vp, vp, vp, vp]
    L.trimkv_paged_move.argtypes = [i32, pc, i32, i64, vp, vp, vp, vp, vp]      # pc: trimkv_paged_rows*, PagedRows array or its bytes
    L.trimkv_paged_sparse_attention.argtypes = [pc, i32, i64, i32, vp, i64, vp, vp, vp, i32, f32, i32, i32, i32, vp, vp, vp,
                                                sz, vp, vp]
    for name in ("trimkv_create_ex", "trimkv_reset", "trimkv_set_gate", "trimkv_set_shared_projection", "trimkv_gate",
                 "trimkv_append", "trimkv_score_and_evict", "trimkv_decode_attention", "trimkv_decode_step_all",
                 "trimkv_get_lengths", "trimkv_get_kept", "trimkv_get_pool", "trimkv_get_select_stats",
                 "trimkv_sync_status", "trimkv_profile", "trimkv_profile_read", "trimkv_select_topk",
                 "trimkv_select_topk_static", "trimkv_set_overlap", "trimkv_set_horizon", "trimkv_set_test_hooks",
                 "trimkv_shard_sample_cap", "trimkv_shard_sample", "trimkv_shard_bracket", "trimkv_shard_filter",
                 "trimkv_shard_candidates", "trimkv_shard_resolve", "trimkv_shard_hist", "trimkv_shard_digit",
                 "trimkv_shard_mark", "trimkv_shard_compact"):
        getattr(L, name).restype = i32
    _lib = L
    return L


def last_error() -> str:
    return lib().trimkv_last_error().decode("utf-8", "replace")


def kernel_launches() -> int:
    return int(lib().trimkv_kernel_launches())


def _check(status: int):
    if status != OK:
        raise TrimkvError(status, last_error())


def _ptr(t: Optional[torch.Tensor], dtype=None, cuda=True):
    if t is None:
        return None
    if cuda and not t.is_cuda:
        raise ValueError("expected a CUDA tensor")
    if not t.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"expected dtype {dtype}, got {t.dtype}")
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


class TrimKV:
    """One budgeted, paged KV cache for a fixed batch of sequences (see include/trimkv.h)."""

    def __init__(self, budget_entries: int, layers: int, kv_heads: int, head_dim: int, *, q_heads: Optional[int] = None,
                 hidden: int = 0, batch: int = 1, gate_hidden: int = 512, gate_embed: int = 64, horizon: int = 2,
                 kv_dtype: str = "bf16", max_chunk: int = 512, max_pool_pages: int = 0, distrust_sample: bool = False,
                 retention_bias: bool = False, per_pool_budget: int = 0, shard_total_layers: int = 0, shard_layer0: int = 0):
        L = lib()
        cfg = Config()
        L.trimkv_default_config(C.byref(cfg), budget_entries, layers, kv_heads, head_dim)
        cfg.q_heads = q_heads if q_heads is not None else kv_heads
        cfg.hidden = hidden
        cfg.max_batch = batch
        cfg.gate_hidden = gate_hidden
        cfg.gate_embed = gate_embed
        cfg.horizon = horizon
        cfg.kv_dtype = {"bf16": DTYPE_BF16, "f32": DTYPE_F32}[kv_dtype]
        cfg.max_chunk = max_chunk
        cfg.max_pool_pages = max_pool_pages
        cfg.retention_bias = 1 if retention_bias else 0
        cfg.per_pool_budget = per_pool_budget
        cfg.shard_total_layers = shard_total_layers
        cfg.shard_layer0 = shard_layer0
        cfg.reserved = 0
        self.cfg = cfg
        self.torch_dtype = torch.bfloat16 if kv_dtype == "bf16" else torch.float32
        self.B, self.L, self.H, self.Hq, self.d, self.D = batch, layers, kv_heads, cfg.q_heads, head_dim, hidden
        h = C.c_void_p()
        _check(L.trimkv_create_ex(C.byref(cfg), C.byref(h)))
        self._h = h
        if distrust_sample:                            # testing aid: forces the selection's exact redo path
            self.set_test_hooks(TEST_DISTRUST_SAMPLE)

    @classmethod
    def from_workload(cls, w, **overrides) -> "TrimKV":
        kw = dict(q_heads=w.q_heads, hidden=w.hidden, batch=w.batch, gate_hidden=w.gate_hidden, gate_embed=w.gate_embed,
                  horizon=w.horizon, kv_dtype=w.kv_dtype, max_chunk=w.chunk)
        kw.update(overrides)
        return cls(w.budget_entries, w.layers, w.kv_heads, w.head_dim, **kw)

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            lib().trimkv_destroy(self._h)
            self._h = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    # ---- gate
    def set_gate(self, layer: int, W1, b1, W2, b2):
        f = torch.float32
        _check(lib().trimkv_set_gate(self._h, layer, _ptr(W1, f), _ptr(b1, f), _ptr(W2, f), _ptr(b2, f)))

    def set_shared_projection(self, w_g, b_g: float):
        _check(lib().trimkv_set_shared_projection(self._h, _ptr(w_g, torch.float32), float(b_g)))

    def gate(self, layer: int, x: torch.Tensor):
        """x [B, n, D] fp32 -> (beta, lambda, c), each [B, n, H] fp32."""
        n = x.shape[1]
        outs = [torch.empty(self.B, n, self.H, device=x.device, dtype=torch.float32) for _ in range(3)]
        _check(lib().trimkv_gate(self._h, layer, n, _ptr(x, torch.float32), _ptr(outs[0]), _ptr(outs[1]), _ptr(outs[2]),
                                 _stream()))
        return tuple(outs)

    # ---- cache
    def append(self, layer: int, k, v, x=None, lam=None, c=None):
        n = k.shape[1]
        f = torch.float32
        _check(lib().trimkv_append(self._h, layer, n, _ptr(x, f), _ptr(lam, f), _ptr(c, f), _ptr(k, self.torch_dtype),
                                   _ptr(v, self.torch_dtype), _stream()))

    def score_and_evict(self):
        _check(lib().trimkv_score_and_evict(self._h, _stream()))

    def decode_attention(self, layer: int, q, out=None):
        if out is None:
            out = torch.empty_like(q)
        _check(lib().trimkv_decode_attention(self._h, layer, _ptr(q, self.torch_dtype), _ptr(out, self.torch_dtype),
                                             _stream()))
        return out

    def prefill_attention(self, layer: int, q, out=None):
        """q [B, n, Hq, d]: causal attention of the n-token chunk just appended to `layer`."""
        if out is None:
            out = torch.empty_like(q)
        _check(lib().trimkv_prefill_attention(self._h, layer, q.shape[1], _ptr(q, self.torch_dtype),
                                              _ptr(out, self.torch_dtype), _stream()))
        return out

    def decode_step_all(self, k, v, q, out, x=None, lam=None):
        f = torch.float32
        _check(lib().trimkv_decode_step_all(self._h, _ptr(x, f), _ptr(lam, f), _ptr(k, self.torch_dtype),
                                            _ptr(v, self.torch_dtype), _ptr(q, self.torch_dtype),
                                            _ptr(out, self.torch_dtype), _stream()))
        return out

    def decode_step_all_host(self, k, v, q, out, x=None, lam=None):
        """Same step with HOST tensors (pinned for asynchronous copies); `out` is a host tensor as well."""
        f = torch.float32
        _check(lib().trimkv_decode_step_all_host(self._h, _ptr(x, f, cuda=False), _ptr(lam, f, cuda=False),
                                                 _ptr(k, self.torch_dtype, cuda=False), _ptr(v, self.torch_dtype, cuda=False),
                                                 _ptr(q, self.torch_dtype, cuda=False), _ptr(out, self.torch_dtype, cuda=False),
                                                 _stream()))
        return out

    def reset(self):
        _check(lib().trimkv_reset(self._h))

    def sync_status(self):
        _check(lib().trimkv_sync_status(self._h))

    def check_invariants(self):
        """Self-check of the cache's bookkeeping (raises TrimkvError E_STATE naming the violated rules)."""
        _check(lib().trimkv_check_invariants(self._h))

    PHASES = ["gate", "append", "h2d_kvq", "attn_main", "d2h_out", "select", "compact", "h2d_x"]

    def profile(self, enable):
        """False/0 off, True/1 every phase, 2 the attention kernel alone."""
        _check(lib().trimkv_profile(self._h, int(enable)))

    def set_horizon(self, horizon: int):
        """New horizon T - t for stored and future entries (0 = infinite)."""
        _check(lib().trimkv_set_horizon(self._h, int(horizon), _stream()))

    def set_test_hooks(self, flags: int):
        """Testing aids of this handle (TEST_* flags; 0 = normal operation)."""
        _check(lib().trimkv_set_test_hooks(self._h, int(flags)))

    def step_stream(self) -> "torch.cuda.ExternalStream":
        """The handle's highest-priority stream as a torch stream: decode steps enqueued on it skip two stream hand-offs."""
        return torch.cuda.ExternalStream(int(lib().trimkv_step_stream(self._h)))

    def set_overlap(self, enable: bool):
        _check(lib().trimkv_set_overlap(self._h, 1 if enable else 0))

    def profile_read(self):
        """{phase: (total ms, intervals)} recorded since profiling was enabled."""
        ms = (C.c_double * 8)()
        cnt = (C.c_int64 * 8)()
        _check(lib().trimkv_profile_read(self._h, ms, cnt))
        return {name: (ms[i], cnt[i]) for i, name in enumerate(self.PHASES)}

    # ---- read-back (synchronising)
    def lengths(self) -> torch.Tensor:
        out = torch.empty(self.B, self.L, self.H, dtype=torch.int32)
        _check(lib().trimkv_get_lengths(self._h, C.c_void_p(out.data_ptr())))
        return out

    def kept(self, seq: int, layer: int, head: int, cap: int) -> torch.Tensor:
        out = torch.empty(max(cap, 1), dtype=torch.int32)
        n = C.c_int(0)
        _check(lib().trimkv_get_kept(self._h, seq, layer, head, C.c_void_p(out.data_ptr()), cap, C.byref(n)))
        return out[: n.value].clone()

    def pool(self, seq: int, layer: int, head: int, cap: int, with_kv: bool = True):
        pos = torch.empty(max(cap, 1), dtype=torch.int32)
        lam = torch.empty(max(cap, 1), dtype=torch.float32)
        c = torch.empty(max(cap, 1), dtype=torch.float32)
        k = torch.empty(max(cap, 1), self.d, dtype=self.torch_dtype) if with_kv else None
        v = torch.empty(max(cap, 1), self.d, dtype=self.torch_dtype) if with_kv else None
        n = C.c_int(0)
        _check(lib().trimkv_get_pool(self._h, seq, layer, head, cap, C.byref(n), C.c_void_p(pos.data_ptr()),
                                     C.c_void_p(lam.data_ptr()), C.c_void_p(c.data_ptr()),
                                     C.c_void_p(k.data_ptr()) if with_kv else None,
                                     C.c_void_p(v.data_ptr()) if with_kv else None))
        m = n.value
        return pos[:m], lam[:m], c[:m], (k[:m] if with_kv else None), (v[:m] if with_kv else None)

    def import_pool(self, seq: int, layer: int, head: int, pos, lam, c, k, v):
        """Fills the (empty) pool from host tensors as `pool` returned them (checkpoint resume)."""
        n = int(pos.numel())
        hp = lambda t: C.c_void_p(t.contiguous().data_ptr()) if n else None
        _check(lib().trimkv_import_pool(self._h, seq, layer, head, n, hp(pos), hp(lam), hp(c), hp(k), hp(v)))

    def import_finish(self, tokens: int):
        _check(lib().trimkv_import_finish(self._h, int(tokens)))

    def select_stats(self) -> torch.Tensor:
        out = torch.empty(self.B, 4, dtype=torch.int64)
        _check(lib().trimkv_get_select_stats(self._h, C.c_void_p(out.data_ptr())))
        return out


def set_global_test_hooks(flags: int):
    """Testing aids of the handle-less calls (select_topk, select_topk_static, paged_sparse_attention); 0 = normal operation."""
    _check(lib().trimkv_set_test_hooks(None, int(flags)))


def select_workspace_bytes(n: int) -> int:
    return int(lib().trimkv_select_workspace_bytes(n))


def select_topk(scores: torch.Tensor, k_keep: int, keep_bits: Optional[torch.Tensor] = None,
                workspace: Optional[torch.Tensor] = None, status: Optional[torch.Tensor] = None):
    """Keep mask (uint64 words as int64 tensor) of the k_keep largest fp32 scores; ties keep the lower index."""
    n = scores.numel()
    words = (n + 63) // 64
    if keep_bits is None:
        keep_bits = torch.empty(max(words, 1), dtype=torch.int64, device=scores.device)
    need = select_workspace_bytes(n)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=scores.device)
    if status is None:
        status = torch.zeros(1, dtype=torch.int32, device=scores.device)
    _check(lib().trimkv_select_topk(_ptr(scores, torch.float32), n, k_keep, _ptr(keep_bits), _ptr(workspace),
                                    workspace.numel(), _ptr(status), _stream()))
    return keep_bits, status


SELECT_STATIC_MAX_N = 1 << 22


def select_topk_static(scores: torch.Tensor, k_keep: int, keep_bits: torch.Tensor, status: torch.Tensor):
    """trimkv_select_topk_static: the same selection, for callers that cannot allocate device memory when
    they call (a serving loop with a fixed memory plan, a framework that bans cudaMalloc after start-up).
    The scratch lives inside the library; the caller passes every buffer: keep_bits (int64 words,
    ceil(n / 64) of them) and status (int32[1]).  At most SELECT_STATIC_MAX_N scores.  Calls share the
    scratch, so do not let two of them overlap on the GPU."""
    n = scores.numel()
    _check(lib().trimkv_select_topk_static(_ptr(scores, torch.float32), n, k_keep, _ptr(keep_bits), _ptr(status),
                                           _stream()))
    return keep_bits, status


# ---- the caller-owned paged cache (trimkv_paged_*): see include/trimkv.h for the layouts
PAGE_SIZE = 64
_KV_DTYPES = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}


# (These calls are short and a decode step makes several, so the checks are made with few attribute reads each.)
def _ints(index: int, name: str, t: torch.Tensor, n: int) -> int:
    """Address of n contiguous int32 on device `index`."""
    if t.dtype is torch.int32 and t.get_device() == index and t.numel() == n and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name}: expected {n} contiguous int32 on cuda:{index}, got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _on(index: int, name: str, t: torch.Tensor, dtype, shape) -> int:
    """Address of a contiguous tensor of device `index`, type and shape."""
    if t.dtype is dtype and t.get_device() == index and t.shape == shape and t.is_contiguous():
        return t.data_ptr()
    raise ValueError(f"{name}: expected a contiguous {dtype} tensor {tuple(shape)} on cuda:{index}, "
                     f"got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _rows(index: int, name: str, t: torch.Tensor, dtype, heads: int, d: int):
    """(address, elements between tokens, tokens) of a [tokens, heads, d] tensor whose rows [heads, d] are contiguous."""
    if t.dim() == 3 and t.dtype is dtype and t.get_device() == index:
        n, h, e = t.shape
        step, sh, sd = t.stride()
        if h == heads and e == d and (n == 0 or ((sd == 1 or d == 1) and (sh == d or heads == 1))):
            return t.data_ptr(), (step if n > 1 else heads * d), n
    raise ValueError(f"{name}: expected {dtype} [tokens, {heads}, {d}] on cuda:{index}, the {heads} x {d} values of a token contiguous, "
                     f"got {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}")


def _small(**numbers):
    """Numbers that the call takes as 32 bits (ctypes would cut a larger one down without a word)."""
    for name, x in numbers.items():
        if not -(1 << 31) <= x < 1 << 31:
            raise ValueError(f"{name} = {x} is out of range")


_pack_cache = struct.Struct("PPPiiiiii").pack      # PagedCache, field by field


def _paged_cache(k_pages, v_pages, key_bounds):
    """(trimkv_paged_cache as bytes, device, dtype, kv_heads, head_dim)"""
    index, dt, shape = k_pages.get_device(), k_pages.dtype, k_pages.shape
    if index < 0:
        raise ValueError("expected a CUDA tensor")
    if len(shape) != 4 or dt not in _KV_DTYPES:
        raise ValueError("k_pages: expected bf16 or fp32 [n_pages, kv_heads, 64, head_dim]")
    n, h, page, d = shape
    return _pack_cache(_on(index, "k_pages", k_pages, dt, shape), _on(index, "v_pages", v_pages, dt, shape),
                       0 if key_bounds is None else _on(index, "key_bounds", key_bounds, dt, (n, h, 2, d)),
                       n, h, d, _KV_DTYPES[dt], page, 0), index, dt, h, d


# The raw handle of a device's current stream and the current device's number, without the wrapper objects where torch
# offers them so: a decode step makes several of these short calls.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _launch(fn, index: int, *args):
    """Calls fn(*args, stream) with device `index` current (the library launches on the current device)."""
    if _current_device() == index:
        status = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, _raw_stream(index))
    if status != OK:
        _check(status)


def paged_plan(old_lens, keep_lens, new_lens, block_table, free_pages, free_count, free_count_out, lens_out, cu_new, slot_map,
               positions=None, status=None):
    """Block tables and slot maps from request lengths (trimkv_paged_plan).  int32 tensors: old_lens, keep_lens (or None),
    new_lens, lens_out [R], block_table [R, W], free_pages [n_pages], free_count and free_count_out [1], cu_new [R + 1],
    slot_map and positions (or None) [max_tokens], status [1].  Works in place; returns nothing.  Every page has one holder here: a
    table whose rows share pages, or for which page_refs are kept, is changed by paged_share and paged_compact alone."""
    n = old_lens.get_device()
    if n < 0:
        raise ValueError("expected a CUDA tensor")
    r, m, pages = old_lens.numel(), slot_map.numel(), free_pages.numel()
    rows, w = block_table.shape
    if rows != r:
        raise ValueError(f"block_table: expected {r} rows, got {rows}")
    _launch(lib().trimkv_paged_plan, n, r, _ints(n, "old_lens", old_lens, r),
            None if keep_lens is None else _ints(n, "keep_lens", keep_lens, r), _ints(n, "new_lens", new_lens, r),
            _ints(n, "block_table", block_table, r * w), w, _ints(n, "free_pages", free_pages, pages), pages,
            _ints(n, "free_count", free_count, 1), _ints(n, "free_count_out", free_count_out, 1), m,
            _ints(n, "lens_out", lens_out, r), _ints(n, "cu_new", cu_new, r + 1), _ints(n, "slot_map", slot_map, m),
            None if positions is None else _ints(n, "positions", positions, m),
            None if status is None else _ints(n, "status", status, 1))


def paged_append(k_pages, v_pages, k, v, slot_map, key_bounds=None, status=None):
    """Writes k and v [tokens, H, d] (rows may be strided) to the slots of slot_map [tokens] (trimkv_paged_append)."""
    cache, n, dt, h, d = _paged_cache(k_pages, v_pages, key_bounds)
    kp, ks, t = _rows(n, "k", k, dt, h, d)
    vp, vs, tv = _rows(n, "v", v, dt, h, d)
    if tv != t:
        raise ValueError("k and v hold different numbers of tokens")
    _launch(lib().trimkv_paged_append, n, cache, t, kp, ks, vp, vs, _ints(n, "slot_map", slot_map, t),
            None if status is None else _ints(n, "status", status, 1))


def paged_workspace_bytes(q_heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().trimkv_paged_workspace_bytes(q_heads, kv_heads, head_dim))


def _paged_batch(n, dt, h, d, q, cu_new, lens, block_table, scale, out, workspace, status, workspace_bytes=paged_workspace_bytes):
    if q.dim() != 3:
        raise ValueError("q: expected [tokens, q_heads, head_dim]")
    shape = q.shape
    hq = shape[1]
    qp, qs, t = _rows(n, "q", q, dt, hq, d)
    r = lens.numel()
    rows, w = block_table.shape
    if rows != r:
        raise ValueError(f"block_table: expected {r} rows, got {rows}")
    if out is None:
        out = torch.empty(shape, dtype=dt, device=q.device)
    if workspace is None:
        workspace = torch.empty(max(256, workspace_bytes(hq, h, d)), dtype=torch.uint8, device=q.device)
    size = workspace.numel()
    batch = (qp, qs, _ints(n, "cu_new", cu_new, r + 1), _ints(n, "lens", lens, r), _ints(n, "block_table", block_table, r * w), w,
             d ** -0.5 if scale is None else scale)
    tail = (_on(n, "out", out, dt, shape), _on(n, "workspace", workspace, torch.uint8, (size,)), size,
            None if status is None else _ints(n, "status", status, 1))
    return r, t, hq, batch, tail, out


def paged_attention(k_pages, v_pages, q, cu_new, lens, block_table, max_new: int = 0, *, scale: Optional[float] = None,
                    window: int = 0, out=None, workspace=None, status=None):
    """Causal attention of the new tokens q [tokens, Hq, d] over a caller-owned paged cache (trimkv_paged_attention)."""
    _small(max_new=max_new, window=window)
    cache, n, dt, h, d = _paged_cache(k_pages, v_pages, None)
    r, t, hq, batch, tail, out = _paged_batch(n, dt, h, d, q, cu_new, lens, block_table, scale, out, workspace, status)
    _launch(lib().trimkv_paged_attention, n, cache, r, t, max_new, hq, *batch, window, *tail)
    return out


def paged_sparse_attention(k_pages, v_pages, key_bounds, q, cu_new, lens, block_table, top_pages: int, *, sink_pages: int = 0,
                           recent_pages: int = 1, scale: Optional[float] = None, out=None, selected=None, workspace=None,
                           status=None):
    """Attention over the top_pages pages that each token selects by their key bounds (trimkv_paged_sparse_attention).
    Returns (out, selected [tokens, H, top_pages])."""
    _small(top_pages=top_pages, sink_pages=sink_pages, recent_pages=recent_pages)
    cache, n, dt, h, d = _paged_cache(k_pages, v_pages, key_bounds)
    r, t, hq, batch, tail, out = _paged_batch(n, dt, h, d, q, cu_new, lens, block_table, scale, out, workspace, status)
    if selected is None:
        selected = torch.empty((t, h, max(top_pages, 0)), dtype=torch.int32, device=q.device)
    sel = _on(n, "selected", selected, torch.int32, (t, h, top_pages))
    _launch(lib().trimkv_paged_sparse_attention, n, cache, r, t, hq, *batch, top_pages, sink_pages, recent_pages, sel, *tail)
    return out, selected


# ---- the caller-owned paged cache in 4 bits (trimkv_paged4_*)
_pack_cache4 = struct.Struct("PPPPPPiiiii4x").pack      # Paged4CacheFields, field by field


class Paged4Cache:
    """A layer's cache in 4 bits: k_codes, v_codes uint8 [n_pages, H, 64, d / 2], k_scales, v_scales float8_e4m3fn (or their bytes)
    [n_pages, H, 64, d / 16], k_shift, v_shift int32 [H] or None.  Holds the tensors; checked once, here."""

    __slots__ = ("fields", "index", "heads", "head_dim", "tensors")

    def __init__(self, k_codes, k_scales, v_codes, v_scales, k_shift=None, v_shift=None):
        index, shape = k_codes.get_device(), k_codes.shape
        if index < 0:
            raise ValueError("expected a CUDA tensor")
        if len(shape) != 4:
            raise ValueError("k_codes: expected uint8 [n_pages, kv_heads, 64, head_dim / 2]")
        n, h, page, half = shape
        scales = (n, h, page, half // 8)

        def bytes_of(name, t):
            return _on(index, name, t, torch.float8_e4m3fn if t.dtype is torch.float8_e4m3fn else torch.uint8, scales)

        self.fields = _pack_cache4(_on(index, "k_codes", k_codes, torch.uint8, shape), bytes_of("k_scales", k_scales),
                                   _on(index, "v_codes", v_codes, torch.uint8, shape), bytes_of("v_scales", v_scales),
                                   0 if k_shift is None else _ints(index, "k_shift", k_shift, h),
                                   0 if v_shift is None else _ints(index, "v_shift", v_shift, h), n, h, 2 * half, page, 0)
        self.index, self.heads, self.head_dim = index, h, 2 * half
        self.tensors = (k_codes, k_scales, v_codes, v_scales, k_shift, v_shift)


def _value_dtype(name, t):
    if t.dtype not in _KV_DTYPES:
        raise ValueError(f"{name}: expected bf16 or fp32, got {t.dtype}")
    return t.dtype


def paged4_append(cache: Paged4Cache, k, v, slot_map, status=None):
    """Rounds k and v [tokens, H, d] (bf16 or fp32, rows may be strided) into the slots of slot_map [tokens] (trimkv_paged4_append)."""
    n, h, d, dt = cache.index, cache.heads, cache.head_dim, _value_dtype("k", k)
    kp, ks, t = _rows(n, "k", k, dt, h, d)
    vp, vs, tv = _rows(n, "v", v, dt, h, d)
    if tv != t:
        raise ValueError("k and v hold different numbers of tokens")
    _launch(lib().trimkv_paged4_append, n, cache.fields, _KV_DTYPES[dt], t, kp, ks, vp, vs, _ints(n, "slot_map", slot_map, t),
            None if status is None else _ints(n, "status", status, 1))


def paged4_read(cache: Paged4Cache, slot_map, k=None, v=None, *, dtype=torch.bfloat16, status=None):
    """The values that the slots of slot_map [n] hold (trimkv_paged4_read): (k, v) [n, H, d]."""
    n, t, device = cache.index, slot_map.numel(), slot_map.device
    if k is not None:
        dtype = _value_dtype("k", k)
    shape = (t, cache.heads, cache.head_dim)
    k = torch.empty(shape, dtype=dtype, device=device) if k is None else k
    v = torch.empty(shape, dtype=dtype, device=device) if v is None else v
    _launch(lib().trimkv_paged4_read, n, cache.fields, _KV_DTYPES[_value_dtype("k", k)], t, _ints(n, "slot_map", slot_map, t), _on(n, "k", k, dtype, shape),
            _on(n, "v", v, dtype, shape), None if status is None else _ints(n, "status", status, 1))
    return k, v


def paged4_workspace_bytes(q_heads: int, kv_heads: int, head_dim: int) -> int:
    return int(lib().trimkv_paged4_workspace_bytes(q_heads, kv_heads, head_dim))


def paged4_attention(cache: Paged4Cache, q, cu_new, lens, block_table, max_new: int = 0, *, scale: Optional[float] = None, window: int = 0,
                     out=None, workspace=None, status=None):
    """Causal attention of the new tokens q [tokens, Hq, d] (bf16 or fp32) over a caller-owned paged cache in 4 bits (trimkv_paged4_attention)."""
    _small(max_new=max_new, window=window)
    n, dt = cache.index, _value_dtype("q", q)
    r, t, hq, batch, tail, out = _paged_batch(n, dt, cache.heads, cache.head_dim, q, cu_new, lens, block_table, scale, out, workspace, status,
                                              paged4_workspace_bytes)
    _launch(lib().trimkv_paged4_attention, n, cache.fields, _KV_DTYPES[dt], r, t, max_new, hq, *batch, window, *tail)
    return out


# ---- rows that share pages, dropped entries, and the rows that move (trimkv_paged_share, _compact, _move)
def _table_pair(n, r, block_table, table_out):
    rows, w = block_table.shape
    if rows != r:
        raise ValueError(f"block_table: expected {r} rows, got {rows}")
    return _ints(n, "block_table", block_table, r * w), _ints(n, "table_out", table_out, r * w), w


def paged_share(source, old_lens, keep_lens, new_lens, block_table, table_out, page_refs, refs_out, free_pages, free_out, free_count,
                free_count_out, lens_out, cu_new, slot_map, positions, move_src, move_dst, move_count, status=None):
    """Forks, growth and release of rows that share pages (trimkv_paged_share).  int32 tensors: source, old_lens, keep_lens, new_lens,
    lens_out [R], block_table and table_out [R, W], page_refs, refs_out, free_pages, free_out [n_pages], free_count, free_count_out,
    move_count, status [1], cu_new [R + 1], slot_map and positions (or None) [max_tokens], move_src and move_dst [max_moves].  A table of
    paged_plan's goes over with counts of 1; paged_plan is not called on it any more."""
    n = old_lens.get_device()
    if n < 0:
        raise ValueError("expected a CUDA tensor")
    r, m, pages, moves = old_lens.numel(), slot_map.numel(), free_pages.numel(), move_src.numel()
    table, out, w = _table_pair(n, r, block_table, table_out)
    _launch(lib().trimkv_paged_share, n, r, _ints(n, "source", source, r), _ints(n, "old_lens", old_lens, r), _ints(n, "keep_lens", keep_lens, r),
            _ints(n, "new_lens", new_lens, r), table, out, w, _ints(n, "page_refs", page_refs, pages), _ints(n, "refs_out", refs_out, pages),
            _ints(n, "free_pages", free_pages, pages), _ints(n, "free_out", free_out, pages), pages, _ints(n, "free_count", free_count, 1),
            _ints(n, "free_count_out", free_count_out, 1), m, _ints(n, "lens_out", lens_out, r), _ints(n, "cu_new", cu_new, r + 1),
            _ints(n, "slot_map", slot_map, m), None if positions is None else _ints(n, "positions", positions, m), moves,
            _ints(n, "move_src", move_src, moves), _ints(n, "move_dst", move_dst, moves), _ints(n, "move_count", move_count, 1),
            None if status is None else _ints(n, "status", status, 1))


def paged_compact(lens, keep_bits, block_table, table_out, page_refs, refs_out, free_pages, free_out, free_count, free_count_out, lens_out,
                  move_src, move_dst, move_count, status=None):
    """Rows without the entries whose bits in keep_bits (int64 [R, W]) are clear (trimkv_paged_compact).  int32 tensors as in
    paged_share; page_refs and refs_out may both be None where no page has two holders.  Entries are renumbered: positions of later calls, and
    windows, count those that are left."""
    n = lens.get_device()
    if n < 0:
        raise ValueError("expected a CUDA tensor")
    r, pages, moves = lens.numel(), free_pages.numel(), move_src.numel()
    table, out, w = _table_pair(n, r, block_table, table_out)
    _launch(lib().trimkv_paged_compact, n, r, _ints(n, "lens", lens, r), _on(n, "keep_bits", keep_bits, torch.int64, (r, w)), table, out, w,
            None if page_refs is None else _ints(n, "page_refs", page_refs, pages), None if refs_out is None else _ints(n, "refs_out", refs_out, pages),
            _ints(n, "free_pages", free_pages, pages), _ints(n, "free_out", free_out, pages), pages, _ints(n, "free_count", free_count, 1),
            _ints(n, "free_count_out", free_count_out, 1), _ints(n, "lens_out", lens_out, r), moves, _ints(n, "move_src", move_src, moves),
            _ints(n, "move_dst", move_dst, moves), _ints(n, "move_count", move_count, 1), None if status is None else _ints(n, "status", status, 1))


_pack_rows = struct.Struct("PPiiii").pack       # PagedRows, field by field


def paged_move(arrays, move_src, move_dst, move_count, key_bounds=None, status=None):
    """Copies rows move_src to rows move_dst [max_moves], the first move_count [1] pairs, in every array (trimkv_paged_move).  arrays: contiguous
    tensors [n_pages, H, 64, ...] of any type, of all layers; key_bounds: per array None or its bounds [n_pages, H, 2, d], or None."""
    n = move_src.get_device()
    if n < 0:
        raise ValueError("expected a CUDA tensor")
    moves, pages, rows = move_src.numel(), None, []
    if key_bounds is not None and len(key_bounds) != len(arrays):
        raise ValueError(f"key_bounds: expected one entry for each of {len(arrays)} arrays, got {len(key_bounds)}")
    for i, t in enumerate(arrays):
        shape = t.shape
        if len(shape) < 3 or shape[2] != PAGE_SIZE or t.get_device() != n or not t.is_contiguous():
            raise ValueError(f"arrays[{i}]: expected a contiguous tensor [n_pages, kv_heads, {PAGE_SIZE}, ...] on cuda:{n}, got {tuple(shape)} with strides {t.stride()} on {t.device}")
        if pages is None:
            pages = shape[0]
        elif shape[0] != pages:
            raise ValueError(f"arrays[{i}]: expected {pages} pages, got {shape[0]}")
        row = math.prod(shape[3:]) * t.element_size()
        bounds = None if key_bounds is None else key_bounds[i]
        if bounds is None:
            rows.append(_pack_rows(t.data_ptr(), 0, shape[1], row, 0, 0))
        else:
            if t.dtype not in _KV_DTYPES or len(shape) != 4:
                raise ValueError(f"arrays[{i}]: bounds want bf16 or fp32 keys [n_pages, kv_heads, {PAGE_SIZE}, head_dim]")
            rows.append(_pack_rows(t.data_ptr(), _on(n, f"key_bounds[{i}]", bounds, t.dtype, (shape[0], shape[1], 2, shape[3])), shape[1], row,
                                   _KV_DTYPES[t.dtype], 0))
    if pages is None:
        return
    _launch(lib().trimkv_paged_move, n, len(rows), b"".join(rows), pages, moves, _ints(n, "move_src", move_src, moves), _ints(n, "move_dst", move_dst, moves),
            _ints(n, "move_count", move_count, 1), None if status is None else _ints(n, "status", status, 1))
