"""Thin ctypes binding of the C ABI in include/lar.h (same names; argument marshalling only).

Every step of the hot path runs in the CUDA kernels of liblar.so.  There is no fallback: if the
library has not been built (python -m paper_2512_04857_b200.build) loading raises.
PyTorch is used by callers for device memory and streams; this module only needs raw addresses.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
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
_torch = None   # the module, once a call that takes tensors has been made


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


# One step of a model makes a call per layer and operator, so the marshalling below is written for host time: the row
# views are packed as bytes, and the calls go through function objects of their own that take them as plain pointers.
_pack_rows = struct.Struct("=Qqq").pack      # lar_rows_t
_FAST = None


def _fast():
    """The entry points of this section with every pointer argument untyped."""
    global _FAST, _torch
    if _FAST is None:
        import torch
        typed, raw = lib(), C.CDLL(LIB_PATH)
        names = ("lar_rope_table", "lar_rope_rotate", "lar_paged_append_rope", "lar_paged_attn", "lar_append_kv_rope")
        plain = {C.POINTER(t): C.c_void_p for t in (lar_rope_t, lar_rows_t, lar_paged_kv_t)}
        for name in names:
            fn = getattr(raw, name)
            fn.restype, fn.argtypes = C.c_int, [plain.get(a, a) for a in getattr(typed, name).argtypes]
        _torch = torch
        _FAST = raw
    return _FAST


def _require(ok, what):
    if not ok:
        raise LarError(LAR_ERR_INVALID_ARG, what)


def _rows(x, n, heads, d, dtype, dev, what):
    """lar_rows_t of a [n, heads, d] tensor with any token and head stride."""
    st = x.stride()
    if x.shape != (n, heads, d) or st[2] != 1 or x.dtype != dtype or x.get_device() != dev:
        raise LarError(LAR_ERR_INVALID_ARG, f"{what}: a {dtype} tensor [{n}, {heads}, {d}] with a dense innermost dimension "
                       f"on the same GPU is expected, not {x.dtype} {list(x.shape)} on {x.device}")
    return _pack_rows(x.data_ptr(), st[0], st[1])


def _dtype_of(x) -> int:
    _fast()
    if x.dtype == _torch.bfloat16:
        return LAR_BF16
    if x.dtype == _torch.float32:
        return LAR_FP32
    raise LarError(LAR_ERR_INVALID_ARG, f"dtype {x.dtype}")


def _ints(x, n, dev, what):
    """Address of a dense int32 tensor [n] on the GPU dev, or None."""
    if x is None:
        return None
    if x.dtype != _torch.int32 or x.get_device() != dev or x.shape != (n,) or (n > 1 and x.stride(0) != 1):
        raise LarError(LAR_ERR_INVALID_ARG, f"{what}: a dense int32 tensor [{n}] on the same GPU is expected")
    return x.data_ptr()


def _positions(pos, rope, n, dev, what):
    """Address and axis stride of pos, int32 [axes, tokens] (or [tokens] for one axis), dense along the tokens."""
    axes, st = rope.n_axes, pos.stride()
    if pos.dtype != _torch.int32 or pos.get_device() != dev or (n > 1 and st[-1] != 1) or \
            (pos.shape != (axes, n) and (axes != 1 or pos.shape != (n,))):
        raise LarError(LAR_ERR_INVALID_ARG, f"{what}: pos is an int32 tensor [{axes}, {n}] on the same GPU")
    return pos.data_ptr(), st[0] if axes > 1 else n


def _device_of(x) -> int:
    dev = x.get_device()
    if dev < 0:
        raise LarError(LAR_ERR_INVALID_ARG, f"a CUDA tensor is expected, not one on {x.device}")
    return dev


def _call(name, dev, *args):
    """The entry point on the GPU dev and torch's current stream there."""
    fn = getattr(_FAST, name)
    if _torch._C._cuda_getDevice() == dev:
        status = fn(*args, _torch._C._cuda_getCurrentRawStream(dev))
    else:
        with _torch.cuda.device(dev):
            status = fn(*args, _torch._C._cuda_getCurrentRawStream(dev))
    if status != LAR_OK:
        raise LarError(status, name)


def rope_table(rope, pos, cos_sin):
    """cos_sin [rows, head_dim] fp32: what decode_step_rope takes, for the positions pos [axes, rows]."""
    _fast()
    dev, rows = _device_of(cos_sin), cos_sin.shape[0]
    _require(cos_sin.dtype == _torch.float32 and cos_sin.shape == (rows, rope.head_dim) and cos_sin.is_contiguous(),
             "rope_table: cos_sin")
    at, stride = _positions(pos, rope, rows, dev, "rope_table")
    _call("lar_rope_table", dev, C.addressof(rope), at, stride, rows, cos_sin.data_ptr())


def rope_rotate(rope, pos, q, q_out, k=None, k_out=None, inverse=False):
    """Rotates q (and k), [tokens, heads, head_dim] with any token and head strides, by pos [axes, tokens]."""
    code, dt, dev = _dtype_of(q), q.dtype, _device_of(q)
    n, hq, d = q.shape
    _require(d == rope.head_dim and (k is None) == (k_out is None), "rope_rotate: shapes")
    at, stride = _positions(pos, rope, n, dev, "rope_rotate")
    hk = 0 if k is None else k.shape[1]
    _call("lar_rope_rotate", dev, C.addressof(rope), code, at, stride, n, _rows(q, n, hq, d, dt, dev, "rope_rotate: q"),
          _rows(q_out, n, hq, d, dt, dev, "rope_rotate: q_out"), hq,
          None if k is None else _rows(k, n, hk, d, dt, dev, "rope_rotate: k"),
          None if k is None else _rows(k_out, n, hk, d, dt, dev, "rope_rotate: k_out"), hk, int(inverse))


class PagedKV:
    """A paged K/V cache in the caller's tensors.

    k_pool, v_pool  [pages, page_tokens, heads, head_dim] (any strides with a dense innermost dimension; a pool laid out
                    [pages, heads, page_tokens, head_dim] is passed as its transpose(1, 2))
    page_table      int32 [seqs, columns], or [seqs, kv_heads, columns] where every head has pages of its own (the pools
                    then have one head)
    lens            int32 [seqs]: live entries, the tokens of the current chunks included
    status          int32 [1] (None: the object keeps one of its own): takes the status bits, see poll_device_status
    """

    def __init__(self, k_pool, v_pool, page_table, lens, n_kv_heads, status=None):
        import torch
        per_head = page_table.dim() == 3
        _require(k_pool.dim() == 4 and k_pool.shape == v_pool.shape and k_pool.stride() == v_pool.stride() and
                 k_pool.stride(3) == 1 and k_pool.dtype == v_pool.dtype and k_pool.device == v_pool.device, "PagedKV: pools")
        pages, page_tokens, heads, d = k_pool.shape
        _require(heads == (1 if per_head else n_kv_heads), "PagedKV: heads of the pools")
        _require(page_table.dtype == torch.int32 and page_table.device == k_pool.device and page_table.dim() in (2, 3) and
                 page_table.stride(-1) == 1 and (not per_head or page_table.shape[1] == n_kv_heads), "PagedKV: page_table")
        seqs = page_table.shape[0]
        _require(lens.dtype == torch.int32 and lens.device == k_pool.device and tuple(lens.shape) == (seqs,), "PagedKV: lens")
        _require(status is None or (status.dtype in (torch.int32, torch.uint32) and status.device == k_pool.device and
                                    status.numel() == 1), "PagedKV: status")
        if status is None:
            status = torch.zeros(1, dtype=torch.int32, device=k_pool.device)
        self._status = status
        self._keep = (k_pool, v_pool, page_table, lens, status)
        self._set(lar_paged_kv_t(
            C.sizeof(lar_paged_kv_t), _dtype_of(k_pool), seqs, n_kv_heads, d, page_tokens, pages, page_table.shape[-1],
            k_pool.stride(0), k_pool.stride(1), 0 if per_head else k_pool.stride(2), k_pool.data_ptr(), v_pool.data_ptr(),
            page_table.data_ptr(), page_table.stride(0), page_table.stride(1) if per_head else 0, lens.data_ptr(),
            lens.stride(0), _ptr(status)), k_pool.dtype, k_pool.device)

    def _set(self, desc, dtype, device):
        self.desc, self._at, self.dtype, self.device = desc, C.addressof(desc), dtype, device
        self.n_seqs, self.n_kv_heads, self.head_dim = desc.n_seqs, desc.n_kv_heads, desc.head_dim

    @classmethod
    def of_cache(cls, cache: "Cache", layer: int) -> "PagedKV":
        """A layer of the library's own cache (its slab must outlive the object)."""
        import torch
        self, desc = cls.__new__(cls), lar_paged_kv_t()
        _chk(lib().lar_cache_paged_view(cache.handle, layer, desc), "lar_cache_paged_view")
        self._keep, self._status = (cache,), None
        self._set(desc, torch.bfloat16 if cache.cfg.dtype == LAR_BF16 else torch.float32, cache.slab.device)
        return self

    def poll_device_status(self) -> int:
        """Waits for the current stream, returns the status bits since the last poll and clears them: 64 a page or slot outside the
        cache, 4 a wait of the bf16 attention ran into its limit and output rows are not valid (0 = clean)."""
        if self._status is None:
            return self._keep[0].poll_device_status()
        bits = int(self._status.item()) & 0xffffffff
        if bits:
            self._status.zero_()
        return bits

    def append_rope(self, k, v, cu_tokens=None, rope=None, pos=None, q=None, q_out=None):
        """Stores the chunks' keys (rotated by rope at pos [axes, tokens]) and values; q is rotated into q_out."""
        _fast()
        n, hkv, d, dt, dev = k.shape[0], self.n_kv_heads, self.head_dim, self.dtype, _device_of(k)
        _require((rope is None) == (pos is None) and (q is None) == (q_out is None) and dev == self.device.index, "append_rope")
        at, stride = (None, 0) if pos is None else _positions(pos, rope, n, dev, "append_rope")
        hq = 0 if q is None else q.shape[1]
        _call("lar_paged_append_rope", dev, self._at, None if rope is None else C.addressof(rope), at, stride,
              _rows(k, n, hkv, d, dt, dev, "append_rope: k"), _rows(v, n, hkv, d, dt, dev, "append_rope: v"),
              None if q is None else _rows(q, n, hq, d, dt, dev, "append_rope: q"),
              None if q is None else _rows(q_out, n, hq, d, dt, dev, "append_rope: q_out"), hq, n,
              _ints(cu_tokens, self.n_seqs + 1, dev, "append_rope: cu_tokens"))

    def attn_workspace(self, n_q_heads, n_tokens, max_chunk=0, max_len=0):
        """A workspace tensor for attn calls of these sizes and all smaller ones (None where none is used)."""
        import torch
        n = lib().lar_paged_attn_workspace_bytes(self.desc, n_q_heads, n_tokens, max_chunk, max_len)
        return torch.empty(n, dtype=torch.uint8, device=self.device) if n else None

    def attn(self, q, out, cu_tokens=None, causal=True, kv_start=None, softmax_scale=0.0, max_chunk=0, max_len=0,
             workspace=None):
        """Attention of the chunks' queries [tokens, heads, head_dim] over the cache; see lar_paged_attn."""
        _fast()
        n, hq, d, dt, dev = q.shape[0], q.shape[1], self.head_dim, self.dtype, _device_of(q)
        _require(dev == self.device.index, "attn: the cache lies on another GPU")
        ws_at, ws = None, 0
        if workspace is not None:
            _require(workspace.get_device() == dev and workspace.is_contiguous(), "attn: workspace")
            ws_at, ws = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        _call("lar_paged_attn", dev, self._at, _rows(q, n, hq, d, dt, dev, "attn: q"), _rows(out, n, hq, d, dt, dev, "attn: out"),
              hq, n, _ints(cu_tokens, self.n_seqs + 1, dev, "attn: cu_tokens"), _ints(kv_start, self.n_seqs, dev, "attn: kv_start"),
              int(causal), softmax_scale, max_chunk, max_len, ws_at, ws)


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
        _fast()
        n, hq, hkv, d, dt, dev = (self.cfg.batch * n_tokens, self.cfg.n_q_heads, self.cfg.n_kv_heads, self.cfg.head_dim,
                                  k.dtype, _device_of(k))
        _require((rope is None) == (pos is None) and (q is None) == (q_out is None) and _dtype_of(k) == self.cfg.dtype and
                 dev == self.slab.get_device(), "append_kv_rope")
        at, stride = (None, 0) if pos is None else _positions(pos, rope, n, dev, "append_kv_rope")
        _call("lar_append_kv_rope", dev, self.handle, layer, None if rope is None else C.addressof(rope), at, stride,
              _rows(k, n, hkv, d, dt, dev, "append_kv_rope: k"), _rows(v, n, hkv, d, dt, dev, "append_kv_rope: v"),
              None if q is None else _rows(q, n, hq, d, dt, dev, "append_kv_rope: q"),
              None if q is None else _rows(q_out, n, hq, d, dt, dev, "append_kv_rope: q_out"), n_tokens)

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
