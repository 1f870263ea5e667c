"""Thin ctypes binding of the C ABI in include/lar.h (same names; argument marshalling only).

Every step of the hot path runs in the CUDA kernels of liblar.so.  There is no fallback: if the
library has not been built (python -m paper_2512_04857_b200.build) loading raises.
PyTorch is used by callers for device memory and streams; this module only needs raw addresses.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblar.so")

LAR_OK, LAR_ERR_INVALID_ARG, LAR_ERR_BAD_STATE, LAR_ERR_CAPACITY, LAR_ERR_CUDA, LAR_ERR_NOMEM, \
    LAR_ERR_DEVICE_CHECK = range(7)
LAR_BF16, LAR_FP32 = 0, 1
LAR_FLAG_NO_HOST_CHECKS, LAR_FLAG_PDL, LAR_FLAG_SHUFFLE_PAGES, LAR_FLAG_TILE_RANGES = 0x1, 0x2, 0x4, 0x8
LAR_FLAG_SCORE_CACHE_NORM = 0x10
LAR_FLAG_HOST_DEFER_OUT = 0x20
LAR_FLAG_SCORE_ACCUM = 0x40
LAR_FLAG_SLOT_REUSE = 0x80
LAR_FLAG_TEST_STALL = 0x100


class lar_config_t(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("n_layers", C.c_int32), ("batch", C.c_int32),
                ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("cond_len", C.c_int32), ("line_width", C.c_int32),
                ("n_lines", C.c_int32), ("anchor_len", C.c_int32), ("recent_lines", C.c_int32),
                ("budget_lines", C.c_int32), ("softmax_scale", C.c_float), ("page_tokens", C.c_int32),
                ("flags", C.c_uint32), ("kv_splits", C.c_int32), ("warps_per_cta", C.c_int32),
                ("stages", C.c_int32), ("page_seed", C.c_uint32), ("decode_ctas", C.c_int32)]


class lar_plan_t(C.Structure):
    _fields_ = [("capacity", C.c_int32), ("pages_per_unit", C.c_int32), ("page_tokens", C.c_int32),
                ("mid_len", C.c_int32), ("kv_splits", C.c_int32), ("warps_per_cta", C.c_int32),
                ("stages", C.c_int32), ("decode_smem_bytes", C.c_int32), ("line_end_smem_bytes", C.c_int32),
                ("compressing", C.c_int32), ("slab_bytes", C.c_uint64), ("decode_ctas", C.c_int32),
                ("max_segments", C.c_int32), ("scratch_bytes", C.c_uint64)]


class lar_rope_t(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("head_dim", C.c_int32), ("n_axes", C.c_int32),
                ("axis_pairs", C.c_int32 * 4), ("interleaved", C.c_int32), ("restart", C.c_int32),
                ("theta", C.c_double)]


class lar_rows_t(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class lar_paged_kv_t(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("dtype", C.c_int32), ("n_seqs", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("page_tokens", C.c_int32), ("n_pages", C.c_int32), ("table_cols", C.c_int32),
                ("page_stride", C.c_int64), ("row_stride", C.c_int64), ("head_stride", C.c_int64),
                ("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("page_table", C.c_void_p),
                ("table_seq_stride", C.c_int64), ("table_head_stride", C.c_int64), ("lens", C.c_void_p),
                ("lens_stride", C.c_int64), ("status", C.c_void_p)]


class LarError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        msg = lib().lar_status_str(status).decode()
        extra = f" (cudaError {lib().lar_last_cuda_error()})" if status == LAR_ERR_CUDA else ""
        super().__init__(f"{what}: {msg}{extra}")


_LIB = None


def lib():
    """Load liblar.so (once).  Raises if the CUDA library has not been built."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2512_04857_b200.build` "
                           "(there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    vp, ip, cfgp, planp = C.c_void_p, C.c_int, C.POINTER(lar_config_t), C.POINTER(lar_plan_t)
    ropep, rowsp, kvp = C.POINTER(lar_rope_t), C.POINTER(lar_rows_t), C.POINTER(lar_paged_kv_t)
    sigs = {
        "lar_plan_query": (C.c_int, [cfgp, planp]),
        "lar_cache_slab_bytes": (C.c_size_t, [cfgp]),
        "lar_cache_create": (C.c_int, [cfgp, vp, C.c_size_t, C.POINTER(vp)]),
        "lar_cache_reset": (C.c_int, [vp, vp]),
        "lar_append_kv": (C.c_int, [vp, ip, vp, vp, ip, vp]),
        "lar_decode_attn": (C.c_int, [vp, ip, vp, vp, vp]),
        "lar_decode_step": (C.c_int, [vp, ip, vp, vp, vp, vp, vp]),
        "lar_decode_step_strided": (C.c_int, [vp, ip, vp, vp, vp, vp, C.c_int64, C.c_int64, C.c_int64, C.c_int64, vp]),
        "lar_decode_step_rope": (C.c_int, [vp, ip, vp, vp, vp, vp, C.c_int64, C.c_int64, C.c_int64, C.c_int64, vp, ip, vp]),
        "lar_decode_step_host": (C.c_int, [vp, ip, vp, vp, vp, vp, vp]),
        "lar_cache_host_join": (C.c_int, [vp, vp]),
        "lar_line_end_score_evict": (C.c_int, [vp, ip, vp]),
        "lar_line_end_score_evict_all": (C.c_int, [vp, vp]),
        "lar_cache_destroy": (C.c_int, [vp]),
        "lar_cache_get_state": (C.c_int, [vp, ip, vp, vp, vp, vp]),
        "lar_cache_poll_device_status": (C.c_int, [vp, C.POINTER(C.c_uint32), vp]),
        "lar_cache_set_host_checks": (C.c_int, [vp, ip]),
        "lar_cache_launch_count": (C.c_uint64, [vp]),
        "lar_cache_get_plan": (C.c_int, [vp, planp]),
        "lar_attend_dense_noalloc": (C.c_int, [vp, vp, vp, vp, ip, ip, ip, ip, C.c_float, vp]),
        "lar_rope_table": (C.c_int, [ropep, vp, C.c_int64, ip, vp, vp]),
        "lar_rope_rotate": (C.c_int, [ropep, ip, vp, C.c_int64, C.c_int64, rowsp, rowsp, ip, rowsp, rowsp, ip, ip, vp]),
        "lar_paged_append_rope": (C.c_int, [kvp, ropep, vp, C.c_int64, rowsp, rowsp, rowsp, rowsp, ip, C.c_int64, vp, vp]),
        "lar_paged_attn": (C.c_int, [kvp, rowsp, rowsp, ip, C.c_int64, vp, vp, ip, C.c_float, ip, ip, vp, C.c_size_t, vp]),
        "lar_paged_attn_workspace_bytes": (C.c_size_t, [kvp, ip, C.c_int64, ip, ip]),
        "lar_cache_paged_view": (C.c_int, [vp, ip, kvp]),
        "lar_append_kv_rope": (C.c_int, [vp, ip, ropep, vp, C.c_int64, rowsp, rowsp, rowsp, rowsp, ip, vp]),
        "lar_status_str": (C.c_char_p, [C.c_int]),
        "lar_last_cuda_error": (C.c_int, []),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(L, name)
        fn.restype, fn.argtypes = res, args
    _LIB = L
    return L


def make_config(*, n_layers, batch, n_q_heads, n_kv_heads, head_dim, dtype, cond_len, line_width, n_lines,
                anchor_len, recent_lines, budget_lines, softmax_scale=0.0, page_tokens=0, flags=0,
                kv_splits=0, warps_per_cta=0, stages=0, page_seed=0, decode_ctas=0) -> lar_config_t:
    dt = {"bf16": LAR_BF16, "fp32": LAR_FP32}.get(dtype, dtype)
    return lar_config_t(C.sizeof(lar_config_t), n_layers, batch, n_q_heads, n_kv_heads, head_dim, dt,
                        cond_len, line_width, n_lines, anchor_len, recent_lines, budget_lines,
                        float(softmax_scale), page_tokens, flags, kv_splits, warps_per_cta, stages, page_seed,
                        decode_ctas)


def config_from_workload(w, **overrides) -> lar_config_t:
    kw = dict(n_layers=w.n_layers, batch=w.batch, n_q_heads=w.n_q_heads, n_kv_heads=w.n_kv_heads,
              head_dim=w.head_dim, dtype=w.dtype, cond_len=w.cond_len, line_width=w.line_width,
              n_lines=w.n_lines, anchor_len=w.anchor_len, recent_lines=w.recent_lines,
              budget_lines=w.budget_lines)
    kw.update(overrides)
    if getattr(w, "score_norm", "mid") == "cache":
        kw["flags"] = kw.get("flags", 0) | LAR_FLAG_SCORE_CACHE_NORM
    if getattr(w, "score_norm", "mid") == "accum":
        kw["flags"] = kw.get("flags", 0) | LAR_FLAG_SCORE_ACCUM
    return make_config(**kw)


def _chk(status: int, what: str):
    if status != LAR_OK:
        raise LarError(status, what)


def _ptr(x) -> Optional[int]:
    """Raw address of a torch tensor / numpy array / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if hasattr(x, "ctypes"):
        return x.ctypes.data
    raise TypeError(type(x))


# ---- the C entry points, same names --------------------------------------------------------------
def lar_plan_query(cfg: lar_config_t) -> lar_plan_t:
    plan = lar_plan_t()
    _chk(lib().lar_plan_query(C.byref(cfg), C.byref(plan)), "lar_plan_query")
    return plan


def lar_cache_slab_bytes(cfg: lar_config_t) -> int:
    return int(lib().lar_cache_slab_bytes(C.byref(cfg)))


def lar_cache_create(cfg: lar_config_t, dev_slab, slab_bytes: int) -> int:
    out = C.c_void_p()
    _chk(lib().lar_cache_create(C.byref(cfg), _ptr(dev_slab), slab_bytes, C.byref(out)), "lar_cache_create")
    return out.value


def lar_cache_reset(cache, stream=None):
    _chk(lib().lar_cache_reset(cache, stream), "lar_cache_reset")


def lar_append_kv(cache, layer, k, v, n_tokens, stream=None):
    _chk(lib().lar_append_kv(cache, layer, _ptr(k), _ptr(v), n_tokens, stream), "lar_append_kv")


def lar_decode_attn(cache, layer, q, out, stream=None):
    _chk(lib().lar_decode_attn(cache, layer, _ptr(q), _ptr(out), stream), "lar_decode_attn")


def lar_decode_step(cache, layer, q, k, v, out, stream=None):
    _chk(lib().lar_decode_step(cache, layer, _ptr(q), _ptr(k), _ptr(v), _ptr(out), stream), "lar_decode_step")


def lar_decode_step_strided(cache, layer, q, k, v, out, q_seq_stride, k_seq_stride, v_seq_stride, out_seq_stride,
                            stream=None):
    _chk(lib().lar_decode_step_strided(cache, layer, _ptr(q), _ptr(k), _ptr(v), _ptr(out), q_seq_stride, k_seq_stride,
                                       v_seq_stride, out_seq_stride, stream), "lar_decode_step_strided")


def lar_decode_step_rope(cache, layer, q, k, v, out, q_seq_stride, k_seq_stride, v_seq_stride, out_seq_stride, cos_sin,
                         interleaved, stream=None):
    _chk(lib().lar_decode_step_rope(cache, layer, _ptr(q), _ptr(k), _ptr(v), _ptr(out), q_seq_stride, k_seq_stride,
                                    v_seq_stride, out_seq_stride, _ptr(cos_sin), int(interleaved), stream),
         "lar_decode_step_rope")


def lar_decode_step_host(cache, layer, q, k, v, out, stream=None):
    _chk(lib().lar_decode_step_host(cache, layer, _ptr(q), _ptr(k), _ptr(v), _ptr(out), stream),
         "lar_decode_step_host")


def lar_cache_host_join(cache, stream=None):
    _chk(lib().lar_cache_host_join(cache, stream), "lar_cache_host_join")


def lar_line_end_score_evict(cache, layer, stream=None):
    _chk(lib().lar_line_end_score_evict(cache, layer, stream), "lar_line_end_score_evict")


def lar_line_end_score_evict_all(cache, stream=None):
    _chk(lib().lar_line_end_score_evict_all(cache, stream), "lar_line_end_score_evict_all")


def lar_cache_destroy(cache):
    _chk(lib().lar_cache_destroy(cache), "lar_cache_destroy")


def lar_cache_get_state(cache, layer, lens=None, index_map=None, scores=None, stream=None):
    _chk(lib().lar_cache_get_state(cache, layer, _ptr(lens), _ptr(index_map), _ptr(scores), stream),
         "lar_cache_get_state")


def lar_cache_poll_device_status(cache, stream=None) -> int:
    """Returns the device status bits (0 = clean); does not raise on a recorded check."""
    bits = C.c_uint32(0)
    st = lib().lar_cache_poll_device_status(cache, C.byref(bits), stream)
    if st not in (LAR_OK, LAR_ERR_DEVICE_CHECK):
        raise LarError(st, "lar_cache_poll_device_status")
    return int(bits.value)


def lar_cache_set_host_checks(cache, enabled: bool):
    _chk(lib().lar_cache_set_host_checks(cache, int(bool(enabled))), "lar_cache_set_host_checks")


def lar_cache_launch_count(cache) -> int:
    return int(lib().lar_cache_launch_count(cache))


def lar_cache_get_plan(cache) -> lar_plan_t:
    plan = lar_plan_t()
    _chk(lib().lar_cache_get_plan(cache, C.byref(plan)), "lar_cache_get_plan")
    return plan


def lar_attend_dense_noalloc(q, k, v, out, n_units, group, head_dim, length, softmax_scale=0.0, stream=None):
    """Decode attention over dense bf16 K/V; the split-KV scratch is a static device array of the library."""
    _chk(lib().lar_attend_dense_noalloc(_ptr(q), _ptr(k), _ptr(v), _ptr(out), n_units, group, head_dim, length,
                                        float(softmax_scale), stream), "lar_attend_dense_noalloc")


# ---- rotary positions, paged caches, chunk attention: torch tensors in, the C calls of the same names -----------------
def make_rope(head_dim, axis_pairs, *, theta=10000.0, interleaved=False, restart=False) -> lar_rope_t:
    """axis_pairs: rotated pairs per position axis (1 to 4 of them, summing to head_dim / 2)."""
    pairs = [int(a) for a in axis_pairs]
    if not 1 <= len(pairs) <= 4:
        raise LarError(LAR_ERR_INVALID_ARG, "make_rope")
    return lar_rope_t(C.sizeof(lar_rope_t), head_dim, len(pairs), (C.c_int32 * 4)(*pairs), int(interleaved),
                      int(restart), float(theta))


def _rows(x):
    """lar_rows_t of a [tokens, heads, head_dim] tensor (any token and head stride), or None."""
    if x is None:
        return None
    t, h, e = x.stride()
    if e != 1 and x.shape[2] > 1:
        raise LarError(LAR_ERR_INVALID_ARG, "rows: the innermost dimension is not dense")
    return lar_rows_t(x.data_ptr(), t, h)


def _dtype_of(x) -> int:
    import torch
    try:
        return {torch.bfloat16: LAR_BF16, torch.float32: LAR_FP32}[x.dtype]
    except KeyError:
        raise LarError(LAR_ERR_INVALID_ARG, f"dtype {x.dtype}") from None


def _require(ok, what):
    if not ok:
        raise LarError(LAR_ERR_INVALID_ARG, what)


def _same(x, like, what):
    _require(x is None or (x.dtype == like.dtype and x.device == like.device), f"{what}: dtype or device")


def _ints(x, shape, like, what):
    """A dense int32 tensor of this shape on the device of `like` (or None)."""
    if x is None:
        return
    import torch
    _require(x.dtype == torch.int32 and x.device == like.device and tuple(x.shape) == shape and x.is_contiguous(),
             f"{what}: an int32 tensor {shape} on {like.device} is expected")


def _pos_stride(pos, rope, n_tokens, like, what):
    """pos: int32 [axes, tokens] (or [tokens] for one axis), dense along the tokens; returns the axes' stride."""
    import torch
    _require(pos.dtype == torch.int32 and pos.device == like.device, f"{what}: pos is an int32 tensor on {like.device}")
    shape = tuple(pos.shape) if pos.dim() == 2 else (1,) + tuple(pos.shape)
    _require(shape == (rope.n_axes, n_tokens) and (n_tokens <= 1 or pos.stride(-1) == 1), f"{what}: pos is [axes, tokens]")
    return pos.stride(0) if pos.dim() == 2 and rope.n_axes > 1 else n_tokens


class _on:
    """Makes a tensor's device current for a call and gives the handle of torch's current stream on it."""
    __slots__ = ("dev", "guard")

    def __init__(self, x):
        self.dev = x.device
        self.guard = None

    def __enter__(self):
        import torch
        if self.dev.type != "cuda":
            raise LarError(LAR_ERR_INVALID_ARG, f"a CUDA tensor is expected, not one on {self.dev}")
        if torch.cuda.current_device() != self.dev.index:
            self.guard = torch.cuda.device(self.dev)
            self.guard.__enter__()
        return torch.cuda.current_stream(self.dev).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def rope_table(rope, pos, cos_sin):
    """cos_sin [rows, head_dim] fp32: what decode_step_rope takes, for the positions pos [axes, rows]."""
    import torch
    rows = cos_sin.shape[0]
    _require(cos_sin.dtype == torch.float32 and tuple(cos_sin.shape) == (rows, rope.head_dim) and cos_sin.is_contiguous(),
             "rope_table: cos_sin")
    stride = _pos_stride(pos, rope, rows, cos_sin, "rope_table")
    with _on(cos_sin) as stream:
        _chk(lib().lar_rope_table(rope, pos.data_ptr(), stride, rows, cos_sin.data_ptr(), stream), "lar_rope_table")


def rope_rotate(rope, pos, q, q_out, k=None, k_out=None, inverse=False):
    """Rotates q (and k), [tokens, heads, head_dim] with any token and head strides, by pos [axes, tokens]."""
    n, hq, d = q.shape
    dt = _dtype_of(q)
    for x in (q_out, k, k_out):
        _same(x, q, "rope_rotate")
    _require(q_out.shape == q.shape and d == rope.head_dim and (k is None) == (k_out is None), "rope_rotate: shapes")
    if k is not None:
        _require(k.shape == k_out.shape and k.shape[0] == n and k.shape[2] == d, "rope_rotate: shapes")
    stride = _pos_stride(pos, rope, n, q, "rope_rotate")
    with _on(q) as stream:
        _chk(lib().lar_rope_rotate(rope, dt, pos.data_ptr(), stride, n, _rows(q), _rows(q_out), hq, _rows(k), _rows(k_out),
                                   0 if k is None else k.shape[1], int(inverse), stream), "lar_rope_rotate")


class PagedKV:
    """A paged K/V cache in the caller's tensors.

    k_pool, v_pool  [pages, page_tokens, heads, head_dim] (any strides with a dense innermost dimension; a pool laid out
                    [pages, heads, page_tokens, head_dim] is passed as its transpose(1, 2))
    page_table      int32 [seqs, columns], or [seqs, kv_heads, columns] where every head has pages of its own (the pools
                    then have one head)
    lens            int32 [seqs]: live entries, the tokens of the current chunks included
    """

    def __init__(self, k_pool, v_pool, page_table, lens, n_kv_heads, status=None):
        import torch
        per_head = page_table.dim() == 3
        _same(v_pool, k_pool, "PagedKV")
        _require(k_pool.dim() == 4 and k_pool.shape == v_pool.shape and k_pool.stride() == v_pool.stride() and
                 k_pool.stride(3) == 1, "PagedKV: pools")
        pages, page_tokens, heads, d = k_pool.shape
        _require(heads == (1 if per_head else n_kv_heads), "PagedKV: heads of the pools")
        _require(page_table.dtype == torch.int32 and page_table.device == k_pool.device and page_table.dim() in (2, 3) and
                 page_table.stride(-1) == 1 and (not per_head or page_table.shape[1] == n_kv_heads), "PagedKV: page_table")
        seqs = page_table.shape[0]
        _require(lens.dtype == torch.int32 and lens.device == k_pool.device and tuple(lens.shape) == (seqs,), "PagedKV: lens")
        _require(status is None or (status.dtype in (torch.int32, torch.uint32) and status.device == k_pool.device and
                                    status.numel() == 1), "PagedKV: status")
        self._keep = (k_pool, v_pool, page_table, lens, status)
        self.k_pool = k_pool
        self.n_seqs, self.n_kv_heads, self.head_dim = seqs, n_kv_heads, d
        self.desc = lar_paged_kv_t(
            C.sizeof(lar_paged_kv_t), _dtype_of(k_pool), seqs, n_kv_heads, d, page_tokens, pages, page_table.shape[-1],
            k_pool.stride(0), k_pool.stride(1), 0 if per_head else k_pool.stride(2), k_pool.data_ptr(), v_pool.data_ptr(),
            page_table.data_ptr(), page_table.stride(0), page_table.stride(1) if per_head else 0, lens.data_ptr(),
            lens.stride(0), _ptr(status))

    @classmethod
    def of_cache(cls, cache: "Cache", layer: int) -> "PagedKV":
        """A layer of the library's own cache (its slab must outlive the object)."""
        self = cls.__new__(cls)
        self.desc = lar_paged_kv_t()
        _chk(lib().lar_cache_paged_view(cache.handle, layer, self.desc), "lar_cache_paged_view")
        import torch
        dt = torch.bfloat16 if cache.cfg.dtype == LAR_BF16 else torch.float32
        self._keep = (cache,)
        self.k_pool = torch.empty(0, dtype=dt, device=cache.slab.device)   # dtype and device of the rows
        self.n_seqs, self.n_kv_heads, self.head_dim = cache.cfg.batch, cache.cfg.n_kv_heads, cache.cfg.head_dim
        return self

    def _check_rows(self, what, *xs):
        for x, heads, n in xs:
            if x is not None:
                _same(x, self.k_pool, what)
                _require(tuple(x.shape) == (n, heads, self.head_dim), f"{what}: shapes")

    def append_rope(self, k, v, cu_tokens=None, rope=None, pos=None, q=None, q_out=None):
        """Stores the chunks' keys (rotated by rope at pos [axes, tokens]) and values; q is rotated into q_out."""
        n = k.shape[0]
        hq = 0 if q is None else q.shape[1]
        self._check_rows("append_rope", (k, self.n_kv_heads, n), (v, self.n_kv_heads, n), (q, hq, n), (q_out, hq, n))
        _require((rope is None) == (pos is None) and (q is None) == (q_out is None), "append_rope")
        _ints(cu_tokens, (self.n_seqs + 1,), k, "append_rope: cu_tokens")
        stride = 0 if pos is None else _pos_stride(pos, rope, n, k, "append_rope")
        with _on(k) as stream:
            _chk(lib().lar_paged_append_rope(self.desc, rope, _ptr(pos), stride, _rows(k), _rows(v), _rows(q), _rows(q_out),
                                             hq, n, _ptr(cu_tokens), stream), "lar_paged_append_rope")

    def attn_workspace(self, n_q_heads, n_tokens, max_chunk=0, max_len=0):
        """A workspace tensor for attn calls of these sizes (None where none is used)."""
        import torch
        n = lib().lar_paged_attn_workspace_bytes(self.desc, n_q_heads, n_tokens, max_chunk, max_len)
        return torch.empty(n, dtype=torch.uint8, device=self.k_pool.device) if n else None

    def attn(self, q, out, cu_tokens=None, causal=True, kv_start=None, softmax_scale=0.0, max_chunk=0, max_len=0,
             workspace=None):
        """Attention of the chunks' queries [tokens, heads, head_dim] over the cache; see lar_paged_attn."""
        n, hq = q.shape[0], q.shape[1]
        self._check_rows("attn", (q, hq, n), (out, hq, n))
        _ints(cu_tokens, (self.n_seqs + 1,), q, "attn: cu_tokens")
        _ints(kv_start, (self.n_seqs,), q, "attn: kv_start")
        ws = 0
        if workspace is not None:
            _require(workspace.device == q.device and workspace.is_contiguous(), "attn: workspace")
            ws = workspace.numel() * workspace.element_size()
        with _on(q) as stream:
            _chk(lib().lar_paged_attn(self.desc, _rows(q), _rows(out), hq, n, _ptr(cu_tokens), _ptr(kv_start), int(causal),
                                      float(softmax_scale), max_chunk, max_len, _ptr(workspace), ws, stream),
                 "lar_paged_attn")


class Cache:
    """Owns the device slab (a torch uint8 tensor) and the C handle; methods mirror the C calls."""

    def __init__(self, cfg: lar_config_t, device="cuda:0"):
        import numpy as np
        import torch
        self._np, self._torch = np, torch
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = lar_cache_slab_bytes(cfg)
        if nbytes == 0:
            raise LarError(LAR_ERR_INVALID_ARG, "lar_cache_slab_bytes")
        with torch.cuda.device(self.device):
            self.slab = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.slab.data_ptr()
            self._slab_ptr = (base + 255) // 256 * 256
            torch.cuda.synchronize(self.device)
            self.handle = lar_cache_create(cfg, self._slab_ptr, nbytes)
        self.plan = lar_cache_get_plan(self.handle)
        self.units = cfg.batch * cfg.n_kv_heads

    def _stream(self):
        return self._torch.cuda.current_stream(self.device).cuda_stream

    def close(self):
        if getattr(self, "handle", None):
            lar_cache_destroy(self.handle)
            self.handle = None
            self.slab = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reset(self):
        lar_cache_reset(self.handle, self._stream())

    def append_kv(self, layer, k, v, n_tokens):
        lar_append_kv(self.handle, layer, k, v, n_tokens, self._stream())

    def append_kv_rope(self, layer, k, v, n_tokens, rope=None, pos=None, q=None, q_out=None):
        """The prefill with rotated keys: k, v, q are [batch * n_tokens, heads, head_dim], sequence by sequence."""
        n, hq = self.cfg.batch * n_tokens, self.cfg.n_q_heads
        for x, heads in ((k, self.cfg.n_kv_heads), (v, self.cfg.n_kv_heads), (q, hq), (q_out, hq)):
            if x is not None:
                _require(tuple(x.shape) == (n, heads, self.cfg.head_dim) and _dtype_of(x) == self.cfg.dtype and
                         x.device == k.device, "append_kv_rope: shapes")
        _require((rope is None) == (pos is None) and (q is None) == (q_out is None), "append_kv_rope")
        stride = 0 if pos is None else _pos_stride(pos, rope, n, k, "append_kv_rope")
        with _on(k) as stream:
            _chk(lib().lar_append_kv_rope(self.handle, layer, rope, _ptr(pos), stride, _rows(k), _rows(v), _rows(q),
                                          _rows(q_out), n_tokens, stream), "lar_append_kv_rope")

    def paged_view(self, layer) -> "PagedKV":
        """The layer as a PagedKV: attention of a chunk (the prefix) over it."""
        return PagedKV.of_cache(self, layer)

    def decode_attn(self, layer, q, out):
        lar_decode_attn(self.handle, layer, q, out, self._stream())

    def decode_step(self, layer, q, k, v, out):
        lar_decode_step(self.handle, layer, q, k, v, out, self._stream())

    def decode_step_strided(self, layer, q, k, v, out, q_seq_stride, k_seq_stride, v_seq_stride, out_seq_stride):
        lar_decode_step_strided(self.handle, layer, q, k, v, out, q_seq_stride, k_seq_stride, v_seq_stride,
                                out_seq_stride, self._stream())

    def decode_step_rope(self, layer, q, k, v, out, q_seq_stride, k_seq_stride, v_seq_stride, out_seq_stride, cos_sin,
                         interleaved=False):
        lar_decode_step_rope(self.handle, layer, q, k, v, out, q_seq_stride, k_seq_stride, v_seq_stride, out_seq_stride,
                             cos_sin, interleaved, self._stream())

    def decode_step_host(self, layer, q, k, v, out):
        lar_decode_step_host(self.handle, layer, q, k, v, out, self._stream())

    def host_join(self):
        lar_cache_host_join(self.handle, self._stream())

    def line_end_score_evict(self, layer):
        lar_line_end_score_evict(self.handle, layer, self._stream())

    def line_end_score_evict_all(self):
        lar_line_end_score_evict_all(self.handle, self._stream())

    def set_host_checks(self, enabled):
        lar_cache_set_host_checks(self.handle, enabled)

    def poll_device_status(self) -> int:
        return lar_cache_poll_device_status(self.handle, self._stream())

    def launch_count(self) -> int:
        return lar_cache_launch_count(self.handle)

    def get_state(self, layer, want_scores=False):
        np = self._np
        lens = np.zeros(self.units, dtype=np.int32)
        imap = np.zeros((self.units, self.plan.capacity), dtype=np.int32)
        scores = np.zeros((self.units, max(self.plan.mid_len, 1)), dtype=np.float32) if want_scores else None
        lar_cache_get_state(self.handle, layer, lens, imap, scores, self._stream())
        return (lens, imap, scores) if want_scores else (lens, imap)
