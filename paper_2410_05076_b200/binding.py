"""Thin binding of libtidal.so (same names as include/tidal.h): ctypes, and for the calls whose kernels take only a few
microseconds the C++ of csrc/fast_call.cpp.

Argument marshalling only: every step of the attention path runs in the CUDA
kernels behind the C-ABI. PyTorch supplies device memory and the current
stream. If the shared library is missing and cannot be built, this module's
`load()` raises, and so does the first block-sparse or page call without the
C++ part; there is no fallback of any kind.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
from typing import Optional, Sequence

import torch

from . import build as _build

OK = 0
ERR_INVALID, ERR_UNSUPPORTED, ERR_NOMEM, ERR_CUDA, ERR_TIMEOUT, ERR_INDEX = -1, -2, -3, -4, -5, -6
ERR_TOO_LARGE, ERR_INTERNAL, ERR_PAGES = -7, -8, -9
KV_CONTIG, KV_PAGED = 0, 1
KV_BF16, KV_FP8_E4M3 = 0, 1
SEL_PER_QHEAD, SEL_PER_KVHEAD, SEL_SHARED = 0, 1, 2
LAYER_FULL, LAYER_SELECT, LAYER_SPARSE = 0, 1, 2
ROPE_HALF, ROPE_INTERLEAVED = 0, 1
ROPE_PLAIN, ROPE_LINEAR, ROPE_BASE, ROPE_BANDS, ROPE_RAMP = 0, 1, 2, 3, 4

EXPORTS = [
    "tidal_create", "tidal_destroy", "tidal_workspace_bytes", "tidal_full_attn", "tidal_select_attn",
    "tidal_sparse_attn", "tidal_decode_step", "tidal_decode_step_host", "tidal_device_status",
    "tidal_launch_count", "tidal_strerror", "tidal_sparse_attn_noalloc", "tidal_kv_append",
    "tidal_decode_step_append", "tidal_set_graphs", "tidal_set_output_dtype", "tidal_set_attend_newest",
    "tidal_set_layer_overlap", "tidal_reserve", "tidal_set_select_margin",
    "tidal_page_map", "tidal_kv_write", "tidal_block_bounds", "tidal_block_select", "tidal_block_attn",
    "tidal_rope_frequencies", "tidal_rope_init", "tidal_rope", "tidal_rope_write", "tidal_chunk_attn", "tidal_chunk_weights",
    "tidal_evict_select", "tidal_kv_gather",
]

BLOCK = 16               # positions per block of the block-sparse calls, and per page


class tidal_kv_t(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("kv_layout", C.c_int32),
        ("k", C.c_void_p), ("v", C.c_void_p),
        ("stride_b", C.c_int64), ("stride_pos", C.c_int64), ("stride_head", C.c_int64),
        ("stride_page", C.c_int64),
        ("page_table", C.c_void_p), ("page_size", C.c_int32), ("max_pages_per_seq", C.c_int32),
        ("num_pages", C.c_int32),
        ("ctx_lens", C.c_void_p), ("max_ctx_len", C.c_int32), ("sm_scale", C.c_float),
        ("kv_dtype", C.c_int32), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
    ]


class tidal_rope_t(C.Structure):
    _fields_ = [("rotary_dim", C.c_int32), ("layout", C.c_int32), ("scale", C.c_float), ("reserved", C.c_int32), ("step", C.c_uint64 * 64)]


class TidalError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {strerror(status)} ({status})")


_lib = None
_fast = None             # csrc/fast_call.cpp: the block-sparse and page calls, whose kernels take a few microseconds


def load() -> C.CDLL:
    """Load libtidal.so, building it with nvcc first if it is missing or stale."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB
    if not os.path.exists(path) or _build.is_stale():
        try:
            _build.build()
        except Exception as exc:  # no silent fallback: neither to another implementation nor to an outdated library
            what = "is older than its sources" if os.path.exists(path) else "is missing"
            raise ImportError(f"libtidal.so {what} and could not be rebuilt: {exc}") from exc
    L = C.CDLL(path)
    P, I32, I64 = C.c_void_p, C.c_int32, C.c_int64
    KVP = C.POINTER(tidal_kv_t)
    L.tidal_create.argtypes = [C.POINTER(P), C.c_int, C.c_size_t]
    L.tidal_create.restype = I32
    L.tidal_destroy.argtypes = [P]
    L.tidal_destroy.restype = I32
    L.tidal_workspace_bytes.argtypes = [KVP, I32]
    L.tidal_workspace_bytes.restype = C.c_size_t
    L.tidal_decode_step_append.argtypes = [P, I32, P, KVP, P, P, P, P, I32, I32, P, P, P]
    L.tidal_decode_step_append.restype = I32
    L.tidal_set_attend_newest.argtypes = [P, I32]
    L.tidal_set_attend_newest.restype = I32
    L.tidal_set_output_dtype.argtypes = [P, I32]
    L.tidal_set_output_dtype.restype = I32
    L.tidal_set_layer_overlap.argtypes = [P, I32]
    L.tidal_set_layer_overlap.restype = I32
    L.tidal_set_select_margin.argtypes = [P, C.c_float]
    L.tidal_set_select_margin.restype = I32
    L.tidal_reserve.argtypes = [P, KVP, I32, I32]
    L.tidal_reserve.restype = I32
    L.tidal_set_graphs.argtypes = [P, I32]
    L.tidal_set_graphs.restype = I32
    L.tidal_kv_append.argtypes = [P, KVP, P, P, P]
    L.tidal_kv_append.restype = I32
    L.tidal_full_attn.argtypes = [P, KVP, P, P, P]
    L.tidal_full_attn.restype = I32
    L.tidal_select_attn.argtypes = [P, KVP, P, I32, I32, P, P, P, P, P]
    L.tidal_select_attn.restype = I32
    L.tidal_sparse_attn.argtypes = [P, KVP, P, P, P, I32, I32, P, P]
    L.tidal_sparse_attn.restype = I32
    L.tidal_sparse_attn_noalloc.argtypes = [KVP, P, P, P, I32, I32, P, P]
    L.tidal_sparse_attn_noalloc.restype = I32
    L.tidal_decode_step.argtypes = [P, I32, P, KVP, C.POINTER(P), C.POINTER(P), I32, I32, P, P, P]
    L.tidal_decode_step.restype = I32
    L.tidal_decode_step_host.argtypes = [P, I32, P, KVP, P, P, I32, I32, P]
    L.tidal_decode_step_host.restype = I32
    L.tidal_page_map.argtypes = [P, I32, P, P, P, I32, I32, P, P, P, I32, P, P, P, P]
    L.tidal_page_map.restype = I32
    L.tidal_kv_write.argtypes = [P, KVP, I32, P, P, I64, I64, P, P]
    L.tidal_kv_write.restype = I32
    L.tidal_block_bounds.argtypes = [P, KVP, P, I32, P, I32, P]
    L.tidal_block_bounds.restype = I32
    L.tidal_block_select.argtypes = [P, KVP, P, P, I32, I32, I32, I32, I32, P, P, P]
    L.tidal_block_select.restype = I32
    L.tidal_block_attn.argtypes = [P, KVP, P, P, P, I32, I32, P, P]
    L.tidal_block_attn.restype = I32
    PD, D64 = C.POINTER(C.c_double), C.c_double
    RP = C.POINTER(tidal_rope_t)
    L.tidal_rope_frequencies.argtypes = [I32, D64, I32, D64, D64, D64, D64, PD, PD]
    L.tidal_rope_frequencies.restype = I32
    L.tidal_rope_init.argtypes = [RP, I32, I32, PD, D64]
    L.tidal_rope_init.restype = I32
    L.tidal_rope.argtypes = [P, RP, I32, I32, I32, P, I64, P, I64, P, P, P, C.c_float, P, I64, P, I64, P]
    L.tidal_rope.restype = I32
    L.tidal_rope_write.argtypes = [P, RP, KVP, I32, P, I64, P, I64, P, I64, P, P, P, P, C.c_float, P, I64, P]
    L.tidal_rope_write.restype = I32
    L.tidal_chunk_attn.argtypes = [P, KVP, I32, P, I64, P, I32, I32, I32, P, P, P]
    L.tidal_chunk_attn.restype = I32
    L.tidal_chunk_weights.argtypes = [P, KVP, I32, P, I64, P, I32, I32, I32, I32, P, C.c_float, P, I64, I32, P]
    L.tidal_chunk_weights.restype = I32
    L.tidal_evict_select.argtypes = [P, KVP, P, I64, I32, I32, I32, I32, P, P, P]
    L.tidal_evict_select.restype = I32
    L.tidal_kv_gather.argtypes = [P, KVP, KVP, P, P, I32, I32, P, I64, P, I64, P]
    L.tidal_kv_gather.restype = I32
    L.tidal_device_status.argtypes = [P, P]
    L.tidal_device_status.restype = I32
    L.tidal_launch_count.argtypes = [P]
    L.tidal_launch_count.restype = I64
    L.tidal_strerror.argtypes = [I32]
    L.tidal_strerror.restype = C.c_char_p
    _lib = L
    return L


def _fast_calls():
    """The module of csrc/fast_call.cpp, built with g++ first if it is missing or stale, at the first call that goes through
    it: the other calls need neither it nor what it is built with."""
    global _fast
    if _fast is not None:
        return _fast
    path = _build.fast_path()
    try:
        if _build.fast_is_stale():
            _build.build_fast()
        spec = importlib.util.spec_from_file_location(__package__ + "._fast_call", path)
        fast = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(fast)
    except Exception as exc:  # no silent fallback here either
        raise ImportError(f"{os.path.basename(path)} (csrc/fast_call.cpp) could not be built or loaded: {exc}") from exc
    L = load()
    fast.init(C.sizeof(tidal_kv_t), C.sizeof(tidal_rope_t),
              *[C.cast(f, C.c_void_p).value for f in (L.tidal_page_map, L.tidal_kv_write, L.tidal_block_bounds, L.tidal_block_select, L.tidal_block_attn,
                                                      L.tidal_rope, L.tidal_rope_write, L.tidal_chunk_attn, L.tidal_chunk_weights,
                                                      L.tidal_evict_select, L.tidal_kv_gather)])
    _fast = fast
    return fast


def strerror(status: int) -> str:
    return load().tidal_strerror(status).decode()


def kv_struct(layer) -> tidal_kv_t:
    """Descriptor of one layer's cache from any object with LayerKV's fields. A descriptor is returned as it is, so
    that a caller may build it once (and then keeps the tensors behind it alive)."""
    if isinstance(layer, tidal_kv_t):
        return layer
    s = tidal_kv_t()
    s.batch, s.num_q_heads, s.num_kv_heads, s.head_dim = (
        layer.batch, layer.num_q_heads, layer.num_kv_heads, layer.head_dim)
    paged = layer.page_table is not None
    s.kv_layout = KV_PAGED if paged else KV_CONTIG
    s.k, s.v = layer.k.data_ptr(), layer.v.data_ptr()
    s.stride_b, s.stride_pos, s.stride_head, s.stride_page = (
        layer.stride_b, layer.stride_pos, layer.stride_head, layer.stride_page)
    if paged:
        s.page_table = layer.page_table.data_ptr()
        s.page_size = layer.page_size
        s.max_pages_per_seq = layer.max_pages_per_seq
        s.num_pages = getattr(layer, "num_pages", 0) or layer.keep[0].shape[0]
    s.ctx_lens = layer.ctx_lens.data_ptr()
    s.max_ctx_len = layer.max_ctx_len
    s.sm_scale = layer.sm_scale
    s.kv_dtype = getattr(layer, "kv_dtype", 0)
    if s.kv_dtype:
        s.k_scale = layer.k_scale.data_ptr() if layer.k_scale is not None else None
        s.v_scale = layer.v_scale.data_ptr() if layer.v_scale is not None else None
    return s


def _stream(device: Optional[int] = None) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _check(status: int, what: str) -> None:
    if status != OK:
        raise TidalError(status, what)


def block_bounds_shape(layer) -> tuple:
    """Shape of the bf16 tensor of a cache's key bounds: one entry per physical page of a paged cache, one per 16
    positions of each sequence of a contiguous one (for its max_ctx_len; a larger third dimension is fine)."""
    s = kv_struct(layer)
    if s.kv_layout == KV_PAGED:
        return (s.num_pages, s.num_kv_heads, 2, s.head_dim)
    return (s.batch, s.num_kv_heads, -(-s.max_ctx_len // BLOCK), 2, s.head_dim)


def rope_plan(rotary_dim: int = 128, base: float = 10000.0, layout: int = ROPE_HALF, scaling: int = ROPE_PLAIN, factor: float = 1.0,
              low: float = 1.0, high: float = 4.0, trained_len: float = 8192.0, inv_freq: Optional[Sequence[float]] = None,
              cos_scale: float = 1.0) -> tidal_rope_t:
    """How positions rotate the first rotary_dim channels of a head: frequencies base^(-2 i / rotary_dim), scaled as tidal.h says for
    ROPE_LINEAR, ROPE_BASE, ROPE_BANDS and ROPE_RAMP, or inv_freq (radians per position of each pair) with the factor cos_scale on cosines and
    sines. Made once and passed to rope and rope_write."""
    L, plan, half = load(), tidal_rope_t(), max(rotary_dim // 2, 1)
    freq = (C.c_double * half)()
    if inv_freq is not None:
        if len(inv_freq) != half:
            raise ValueError(f"inv_freq: {half} frequencies are wanted, got {len(inv_freq)}")
        freq[:] = [float(x) for x in inv_freq]
    else:
        s = C.c_double()
        _check(L.tidal_rope_frequencies(rotary_dim, base, scaling, factor, low, high, trained_len, freq, C.byref(s)), "tidal_rope_frequencies")
        cos_scale = s.value
    _check(L.tidal_rope_init(C.byref(plan), rotary_dim, layout, freq, cos_scale), "tidal_rope_init")
    return plan


def sparse_attn_noalloc(layer, q: torch.Tensor, idx: torch.Tensor, idx_count: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """tidal_sparse_attn_noalloc on the current device and stream: sparse attention for callers that
    may not allocate device memory. No context is involved; the library's fixed static scratch is
    used, so batch * num_q_heads is limited to 4096 and overlapping calls on one GPU race. `out`
    should be passed by such callers (this wrapper allocates it with torch only as a convenience)."""
    if out is None:
        out = torch.empty(layer.batch, layer.num_q_heads, layer.head_dim, dtype=torch.float32, device=q.device)
    s = kv_struct(layer)
    _, hi, k = idx.shape
    _check(load().tidal_sparse_attn_noalloc(C.byref(s), q.data_ptr(), idx.data_ptr(),
                                            idx_count.data_ptr() if idx_count is not None else None, k, hi,
                                            out.data_ptr(), _stream()), "tidal_sparse_attn_noalloc")
    return out


class Tidal:
    """A libtidal context on one CUDA device (use one context per stream)."""

    def __init__(self, device: int = 0, workspace_bytes: int = 0):
        self.lib = load()
        self.ctx = C.c_void_p()
        _check(self.lib.tidal_create(C.byref(self.ctx), device, workspace_bytes), "tidal_create")
        self.device = device
        self.out_dtype = torch.float32

    @property
    def _handle(self) -> int:
        return self.ctx.value or 0

    def close(self) -> None:
        if getattr(self, "ctx", None) and self.ctx.value:
            self.lib.tidal_destroy(self.ctx)
            self.ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @staticmethod
    def workspace_bytes(layer, k: int) -> int:
        s = kv_struct(layer)
        return load().tidal_workspace_bytes(C.byref(s), k)

    def reserve(self, layer, k: int, num_layers_host: int = 0) -> None:
        """Allocate everything later calls with this cache shape and budget need (then they can be captured)."""
        s = kv_struct(layer)
        _check(self.lib.tidal_reserve(self.ctx, C.byref(s), k, num_layers_host), "tidal_reserve")

    def kv_append(self, layer, k_new: torch.Tensor, v_new: torch.Tensor) -> None:
        """Write the new token's rows (bf16 [B, Hkv, d]) at position ctx_lens[b] - 1 of the layer's cache."""
        s = kv_struct(layer)
        _check(self.lib.tidal_kv_append(self.ctx, C.byref(s), k_new.data_ptr(), v_new.data_ptr(), _stream()),
               "tidal_kv_append")

    def full_attn(self, layer, q: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        if out is None:
            out = torch.empty(layer.batch, layer.num_q_heads, layer.head_dim, dtype=self.out_dtype, device=q.device)
        s = kv_struct(layer)
        _check(self.lib.tidal_full_attn(self.ctx, C.byref(s), q.data_ptr(), out.data_ptr(), _stream()),
               "tidal_full_attn")
        return out

    def select_attn(self, layer, q: torch.Tensor, k: int, granularity: int = SEL_PER_QHEAD,
                    out: Optional[torch.Tensor] = None, idx: Optional[torch.Tensor] = None,
                    idx_count: Optional[torch.Tensor] = None, scores: Optional[torch.Tensor] = None):
        hi = {SEL_PER_QHEAD: layer.num_q_heads, SEL_PER_KVHEAD: layer.num_kv_heads, SEL_SHARED: 1}.get(granularity, 1)
        if out is None:
            out = torch.empty(layer.batch, layer.num_q_heads, layer.head_dim, dtype=self.out_dtype, device=q.device)
        if idx is None:
            idx = torch.empty(layer.batch, hi, max(k, 1), dtype=torch.int32, device=q.device)
        if idx_count is None:
            idx_count = torch.empty(layer.batch, dtype=torch.int32, device=q.device)
        s = kv_struct(layer)
        _check(self.lib.tidal_select_attn(self.ctx, C.byref(s), q.data_ptr(), k, granularity, out.data_ptr(),
                                          idx.data_ptr(), idx_count.data_ptr(),
                                          scores.data_ptr() if scores is not None else None, _stream()),
               "tidal_select_attn")
        return out, idx, idx_count

    def sparse_attn(self, layer, q: torch.Tensor, idx: torch.Tensor, idx_count: Optional[torch.Tensor] = None,
                    out: Optional[torch.Tensor] = None) -> torch.Tensor:
        if out is None:
            out = torch.empty(layer.batch, layer.num_q_heads, layer.head_dim, dtype=self.out_dtype, device=q.device)
        s = kv_struct(layer)
        _, hi, k = idx.shape
        _check(self.lib.tidal_sparse_attn(self.ctx, C.byref(s), q.data_ptr(), idx.data_ptr(),
                                          idx_count.data_ptr() if idx_count is not None else None, k, hi,
                                          out.data_ptr(), _stream()), "tidal_sparse_attn")
        return out

    def make_step(self, sched: Sequence[int], layers: Sequence, qs: Sequence[torch.Tensor],
                  outs: Sequence[torch.Tensor], k: int, granularity: int = SEL_PER_QHEAD):
        """Marshal the per-layer arrays once; the returned callable enqueues one decode step."""
        L = len(sched)
        sched_arr = (C.c_uint8 * L)(*sched)
        kvs = (tidal_kv_t * L)(*[kv_struct(l) for l in layers])
        qp = (C.c_void_p * L)(*[q.data_ptr() for q in qs])
        op = (C.c_void_p * L)(*[o.data_ptr() for o in outs])
        hi = {SEL_PER_QHEAD: layers[0].num_q_heads, SEL_PER_KVHEAD: layers[0].num_kv_heads, SEL_SHARED: 1}[granularity]
        dev = qs[0].device
        idx = torch.full((layers[0].batch, hi, k), -1, dtype=torch.int32, device=dev)
        cnt = torch.zeros(layers[0].batch, dtype=torch.int32, device=dev)
        keep = (sched_arr, kvs, qp, op, list(layers), list(qs), list(outs))

        def step():
            _check(self.lib.tidal_decode_step(self.ctx, L, sched_arr, kvs, qp, op, k, granularity,
                                              idx.data_ptr(), cnt.data_ptr(), _stream()), "tidal_decode_step")

        step.idx, step.idx_count, step.keep = idx, cnt, keep
        return step

    def decode_step_append(self, sched, layers, qs, k_new, v_new, k: int, granularity: int = SEL_PER_QHEAD):
        """One step including the cache update: k_new[i], v_new[i] (bf16 [B, Hkv, d]) go to position
        ctx_lens[b] - 1 of layer i's cache before the layers run. Returns (outs, idx, idx_count)."""
        L = len(sched)
        outs = [torch.empty(l.batch, l.num_q_heads, l.head_dim, dtype=self.out_dtype, device=qs[0].device)
                for l in layers]
        hi = {SEL_PER_QHEAD: layers[0].num_q_heads, SEL_PER_KVHEAD: layers[0].num_kv_heads, SEL_SHARED: 1}[granularity]
        idx = torch.full((layers[0].batch, hi, k), -1, dtype=torch.int32, device=qs[0].device)
        cnt = torch.zeros(layers[0].batch, dtype=torch.int32, device=qs[0].device)
        ptrs = lambda ts: (C.c_void_p * L)(*[t.data_ptr() for t in ts])
        _check(self.lib.tidal_decode_step_append(
            self.ctx, L, (C.c_uint8 * L)(*sched), (tidal_kv_t * L)(*[kv_struct(l) for l in layers]), ptrs(qs),
            ptrs(k_new), ptrs(v_new), ptrs(outs), k, granularity, idx.data_ptr(), cnt.data_ptr(), _stream()),
            "tidal_decode_step_append")
        return outs, idx, cnt

    def decode_step(self, sched, layers, qs, k: int, granularity: int = SEL_PER_QHEAD):
        outs = [torch.empty(l.batch, l.num_q_heads, l.head_dim, dtype=self.out_dtype, device=qs[0].device)
                for l in layers]
        step = self.make_step(sched, layers, qs, outs, k, granularity)
        step()
        return outs, step.idx, step.idx_count

    def make_step_host(self, sched, layers, q_host: torch.Tensor, out_host: torch.Tensor, k: int,
                       granularity: int = SEL_PER_QHEAD):
        """q_host bf16 [L,B,Hq,d] and out_host fp32 [L,B,Hq,d] in (pinned) host memory."""
        L = len(sched)
        sched_arr = (C.c_uint8 * L)(*sched)
        kvs = (tidal_kv_t * L)(*[kv_struct(l) for l in layers])
        assert q_host.device.type == "cpu" and out_host.device.type == "cpu"
        assert q_host.is_contiguous() and out_host.is_contiguous()

        def step():
            _check(self.lib.tidal_decode_step_host(self.ctx, L, sched_arr, kvs, q_host.data_ptr(),
                                                   out_host.data_ptr(), k, granularity, _stream()),
                   "tidal_decode_step_host")

        step.keep = (sched_arr, kvs, list(layers), q_host, out_host)
        return step

    def set_attend_newest(self, enabled: bool) -> None:
        """Sparse layers also attend the newest token (an optional deviation from the paper's algorithm)."""
        _check(self.lib.tidal_set_attend_newest(self.ctx, 1 if enabled else 0), "tidal_set_attend_newest")

    def set_output_bf16(self, enabled: bool) -> None:
        """Later calls write bf16 outputs (pass bf16 `out` tensors) instead of fp32."""
        _check(self.lib.tidal_set_output_dtype(self.ctx, 1 if enabled else 0), "tidal_set_output_dtype")
        self.out_dtype = torch.bfloat16 if enabled else torch.float32

    def set_graphs(self, enabled: bool) -> None:
        """Record whole steps as CUDA graphs and replay them (on by default; needs a non-default stream)."""
        _check(self.lib.tidal_set_graphs(self.ctx, 1 if enabled else 0), "tidal_set_graphs")

    def set_select_margin(self, margin: float) -> None:
        """Safety factor of the selection layers' provisional thresholds (default 3; 0: rank all scores)."""
        _check(self.lib.tidal_set_select_margin(self.ctx, margin), "tidal_set_select_margin")

    def set_layer_overlap(self, enabled: bool) -> None:
        """Layers of a step may stream their inputs while the layer before them finishes (on by default)."""
        _check(self.lib.tidal_set_layer_overlap(self.ctx, 1 if enabled else 0), "tidal_set_layer_overlap")

    # ---- paged caches filled on the device, block-sparse attention ------------------------------------------------

    # (arguments are checked and the current stream of the context's device is looked up in csrc/fast_call.cpp)

    def page_map(self, old_lens: torch.Tensor, new_lens: torch.Tensor, page_table: torch.Tensor, free_pages: torch.Tensor,
                 num_free: torch.Tensor, slots: torch.Tensor, num_free_out: Optional[torch.Tensor] = None,
                 positions: Optional[torch.Tensor] = None, token_offsets: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Grow and shrink sequences from old_lens to new_lens (int32 [B]): pages are taken from and given back to the
        stack free_pages (int32 [num_pages], num_free (int32, one element) of them valid), page_table (int32 [B, width])
        gets the new entries and slots (int64 [max_tokens]) every new token's place in the cache, -1 behind the
        last. num_free_out receives the new count (default: num_free itself); positions (int32 [max_tokens])
        and token_offsets (int32 [B + 1]) are optional outputs. Returns slots. A request that does not fit changes
        nothing and shows in device_status() as ERR_PAGES."""
        rc = (_fast or _fast_calls()).page_map(self._handle, self.device, old_lens, new_lens, page_table, free_pages, num_free, slots, num_free_out,
                            positions, token_offsets)
        if rc:
            raise TidalError(rc, "tidal_page_map")
        return slots

    def kv_write(self, layer, k_new: torch.Tensor, v_new: torch.Tensor, slots: torch.Tensor) -> None:
        """Write the rows of T tokens (bf16 [T, Hkv, d]; only the two inner dimensions have to be contiguous) at their slots
        (int64 [T]; -1: skipped) of the layer's cache; an FP8 cache quantises them with its scales."""
        rc = (_fast or _fast_calls()).kv_write(self._handle, self.device, kv_struct(layer), k_new, v_new, slots)
        if rc:
            raise TidalError(rc, "tidal_kv_write")

    def block_bounds(self, layer, bounds: Optional[torch.Tensor] = None, start_lens: Optional[torch.Tensor] = None,
                     max_new: int = 0) -> torch.Tensor:
        """Channelwise least and greatest key of every block of 16 positions (bf16, see block_bounds_shape): of all
        blocks, or of those that hold positions from start_lens (int32 [B]) on (of the last one, where a sequence has become
        shorter). max_new: host bound of the tokens that came since start_lens (0: not known)."""
        s = kv_struct(layer)
        if bounds is None:
            bounds = torch.zeros(block_bounds_shape(s), dtype=torch.bfloat16, device=f"cuda:{self.device}")
        rc = (_fast or _fast_calls()).block_bounds(self._handle, self.device, s, bounds, start_lens, max_new)
        if rc:
            raise TidalError(rc, "tidal_block_bounds")
        return bounds

    def block_select(self, layer, bounds: torch.Tensor, q: torch.Tensor, m: int, granularity: int = SEL_PER_QHEAD,
                     keep_first: int = 0, keep_last: int = 0, idx: Optional[torch.Tensor] = None,
                     idx_count: Optional[torch.Tensor] = None):
        """The m blocks per index head with the largest upper bound of their logits, the first keep_first and the last
        keep_last blocks among them. Returns (idx int32 [B, Hi, m] ascending and -1 padded, idx_count int32 [B])."""
        s = kv_struct(layer)
        if idx is None:
            hi = {SEL_PER_QHEAD: s.num_q_heads, SEL_PER_KVHEAD: s.num_kv_heads, SEL_SHARED: 1}.get(granularity, 1)
            idx = torch.empty(s.batch, hi, max(m, 1), dtype=torch.int32, device=q.device)
        if idx_count is None:
            idx_count = torch.empty(s.batch, dtype=torch.int32, device=q.device)
        rc = (_fast or _fast_calls()).block_select(self._handle, self.device, s, bounds, q, m, granularity, keep_first, keep_last, idx, idx_count)
        if rc:
            raise TidalError(rc, "tidal_block_select")
        return idx, idx_count

    def block_attn(self, layer, q: torch.Tensor, idx: torch.Tensor, idx_count: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention over the blocks listed in idx (int32 [B, Hi, m], block_select's or any other)."""
        s = kv_struct(layer)
        if out is None:
            out = torch.empty(s.batch, s.num_q_heads, s.head_dim, dtype=self.out_dtype, device=q.device)
        rc = (_fast or _fast_calls()).block_attn(self._handle, self.device, s, q, idx, idx_count, out, self.out_dtype is torch.bfloat16)
        if rc:
            raise TidalError(rc, "tidal_block_attn")
        return out

    # ---- a prompt's way into the cache: norms and rotary positions, chunk attention, eviction -------------------------

    def rope(self, plan: tidal_rope_t, q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor,
             q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6,
             q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
        """Queries and keys of T tokens (bf16 [T, H, 128]; only the two inner dimensions have to be contiguous) normed per head where a
        weight (bf16 [128]) is given and rotated to their positions (int32 [T]; negative: left unwritten). q_out and k_out may be q
        and k. Returns (q_out, k_out)."""
        if q_out is None and q is not None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        if k_out is None and k is not None:
            k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        rc = (_fast or _fast_calls()).rope(self._handle, self.device, plan, q, k, positions, q_weight, k_weight, eps, q_out, k_out)
        if rc:
            raise TidalError(rc, "tidal_rope")
        return q_out, k_out

    def rope_write(self, layer, plan: tidal_rope_t, q: Optional[torch.Tensor], k_new: torch.Tensor, v_new: torch.Tensor,
                   positions: torch.Tensor, slots: torch.Tensor, q_weight: Optional[torch.Tensor] = None,
                   k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, q_out: Optional[torch.Tensor] = None):
        """rope with the keys, and the values, written at their slots (int64 [T]; -1: skipped) of the layer's cache; an FP8 cache
        quantises them with its scales. Returns q_out (None without q)."""
        if q_out is None and q is not None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        rc = (_fast or _fast_calls()).rope_write(self._handle, self.device, kv_struct(layer), plan, q, k_new, v_new, positions, slots, q_weight,
                                                 k_weight, eps, q_out)
        if rc:
            raise TidalError(rc, "tidal_rope_write")
        return q_out

    def chunk_attn(self, layer, q: torch.Tensor, q_offsets: torch.Tensor, max_new: int = 0, causal: bool = True, window: int = 0,
                   out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of every sequence's newest tokens (q: bf16 [T, Hq, 128], sequence b's rows q_offsets[b] .. q_offsets[b + 1] - 1; the cache
        holds their keys and values already) over all cached positions up to their own, or the last `window` of them. max_new: host bound of
        the tokens of a sequence (0: not known). lse: optional fp32 [T, Hq] output."""
        if out is None:
            out = torch.empty(q.shape, dtype=self.out_dtype, device=q.device)
        rc = (_fast or _fast_calls()).chunk_attn(self._handle, self.device, kv_struct(layer), q, q_offsets, max_new, 1 if causal else 0, window, out,
                                                 self.out_dtype is torch.bfloat16, lse)
        if rc:
            raise TidalError(rc, "tidal_chunk_attn")
        return out

    def chunk_weights(self, layer, q: torch.Tensor, q_offsets: torch.Tensor, lse: torch.Tensor, weights: torch.Tensor, decay: float = 1.0,
                      max_new: int = 0, causal: bool = True, window: int = 0, last: int = 0) -> torch.Tensor:
        """weights (fp32 [B, Hkv or 1, >= max_ctx_len]) = decay * weights + the attention weight that every cached position receives from
        those queries (from the last `last` of each chunk, if > 0); lse is chunk_attn's. A chunk's own positions count as 0 before."""
        rc = (_fast or _fast_calls()).chunk_weights(self._handle, self.device, kv_struct(layer), q, q_offsets, lse, weights, decay, max_new,
                                                    1 if causal else 0, window, last)
        if rc:
            raise TidalError(rc, "tidal_chunk_weights")
        return weights

    def evict_select(self, layer, weights: torch.Tensor, m: int, keep_first: int = 0, keep_last: int = 0, kept: Optional[torch.Tensor] = None,
                     new_lens: Optional[torch.Tensor] = None):
        """The m positions per sequence and weight head with the largest weights, the first keep_first and the last keep_last among them.
        Returns (kept int32 [B, heads, m] ascending and -1 padded, new_lens int32 [B])."""
        s = kv_struct(layer)
        if kept is None:
            kept = torch.empty(s.batch, weights.shape[1], max(m, 1), dtype=torch.int32, device=weights.device)
        if new_lens is None:
            new_lens = torch.empty(s.batch, dtype=torch.int32, device=weights.device)
        rc = (_fast or _fast_calls()).evict_select(self._handle, self.device, s, weights, m, keep_first, keep_last, kept, new_lens)
        if rc:
            raise TidalError(rc, "tidal_evict_select")
        return kept, new_lens

    def kv_gather(self, layer, kept: torch.Tensor, counts: torch.Tensor, into=None, weights: Optional[torch.Tensor] = None,
                  weights_out: Optional[torch.Tensor] = None) -> None:
        """The rows of the listed positions (kept: int32 [B, Hkv or 1, m], counts[b] of them) moved to the front of the layer's cache, or
        copied to the cache `into`; weights along, to weights_out (within the cache: in place by default)."""
        if weights is not None and weights_out is None and into is None:
            weights_out = weights
        rc = (_fast or _fast_calls()).kv_gather(self._handle, self.device, kv_struct(layer), None if into is None else kv_struct(into), kept, counts,
                                                weights, weights_out)
        if rc:
            raise TidalError(rc, "tidal_kv_gather")

    def device_status(self) -> int:
        """Waits for the current stream of the context's device, then returns and clears one kind of what its work has noted
        (OK: nothing is left)."""
        return self.lib.tidal_device_status(self.ctx, _stream(self.device))

    def launch_count(self) -> int:
        return self.lib.tidal_launch_count(self.ctx)
