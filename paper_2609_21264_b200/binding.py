"""ctypes binding of the C ABI in ``include/fa.h`` -- argument marshalling only.

Function names and argument order follow the header.  Pointers are plain
integers (``tensor.data_ptr()``, ``stream.cuda_stream``); `forward` is a small
convenience that takes torch tensors, allocates O and lse with torch (device
memory plumbing) and calls `fa_forward`.  There is no fallback: if the library
is missing or the call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os

from . import build as _build

FA_OK = 0
FA_ERR_INVALID_ARG = 1
FA_ERR_UNSUPPORTED = 2
FA_ERR_CUDA = 3
FA_ERR_DEVICE_TIMEOUT = 4
FA_ERR_NO_DEVICE = 5
FA_ERR_OOM = 6
FA_FLAG_SERIAL_KERNEL = 1
FA_FLAG_DEBUG_DROP_V_LOAD = 2
FA_FLAG_NO_DEPENDENT_LAUNCH = 4
FA_FLAG_NO_PERSISTENT = 8
FA_FLAG_FORCE_PERSISTENT = 16
FA_FLAG_STREAM_KERNEL = 32
FA_FLAG_NO_STREAM_KERNEL = 64
FA_FLAG_NO_HEAD_PACKING = 128
FA_FLAG_LEGACY_PAIR_KERNEL = 256
FA_FLAG_TWO_CTA_KERNEL = 512
FA_FLAG_QUAD_KERNEL = 1024

EXPORTS = ("fa_create", "fa_forward", "fa_forward_strided", "fa_forward_varlen", "fa_forward_fp8", "fa_forward_mxfp8", "fa_plan", "fa_forward_host", "fa_last_status", "fa_destroy",
           "fa_strerror", "fa_launch_count", "fa_last_kernel_name", "fa_last_kv_splits",
           "fa_forward_split_noalloc", "fa_noalloc_scratch_bytes", "fa_noalloc_last_status", "fa_debug_set_drop_v_load",
           "fa_append_paged", "fa_forward_paged", "fa_forward_paged_diff", "fa_forward_diff", "fa_device",
           "fa_plan_paged")
FA_CACHE_BF16 = 0
FA_CACHE_E4M3 = 1
FA_PAGED_MAX_SQ = 16


class FaError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__("%s: %s (status %d)" % (what, fa_strerror(status), status))
        self.status = status


class fa_config(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("device", ctypes.c_int32),
                ("flags", ctypes.c_uint32), ("wait_limit_ms", ctypes.c_uint32),
                ("kv_splits", ctypes.c_uint32), ("scratch_bytes", ctypes.c_uint64)]


class fa_paged_cache(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("type", ctypes.c_int32), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("num_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("dqk", ctypes.c_int32),
                ("dv", ctypes.c_int32), ("reserved", ctypes.c_int32), ("k_strides", ctypes.c_int64 * 3),
                ("v_strides", ctypes.c_int64 * 3), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class fa_paged_seqs(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("B", ctypes.c_int32), ("block_table", ctypes.c_void_p),
                ("table_stride", ctypes.c_int64), ("seq_lens", ctypes.c_void_p), ("max_pages", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class fa_rope(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("max_pos", ctypes.c_int32), ("cos_sin", ctypes.c_void_p),
                ("dim", ctypes.c_int32), ("offset", ctypes.c_int32), ("span", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class fa_diff(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("eps", ctypes.c_float), ("lambda_", ctypes.c_void_p),
                ("weight", ctypes.c_void_p), ("out_scale", ctypes.c_float), ("reserved", ctypes.c_float)]


class fa_paged_plan_info(ctypes.Structure):
    _fields_ = [("rows_per_block", ctypes.c_int32), ("row_blocks", ctypes.c_int32), ("ctas", ctypes.c_int32), ("part_cost", ctypes.c_int32),
                ("units", ctypes.c_int64), ("units_per_cta", ctypes.c_int64), ("pieces", ctypes.c_int64)]


class fa_paged_piece(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("cta", "sequence", "kv_head", "row_block", "first_tile", "end_tile", "slot", "pieces",
                                              "first_cta")]


_I64x2 = ctypes.c_int64 * 2
_I64x3 = ctypes.c_int64 * 3
_I64x4 = ctypes.c_int64 * 4
_I64x8 = ctypes.c_int64 * 8
_I64x12 = ctypes.c_int64 * 12
_SEQS_SIZE = ctypes.sizeof(fa_paged_seqs)
_lib = None


def library_path() -> str:
    return _build.LIB_PATH


class fa_plan_info(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_char_p), ("kv_splits", ctypes.c_int32), ("ctas", ctypes.c_int64),
                ("heads_per_tile", ctypes.c_int32), ("estimate_pair_us", ctypes.c_double), ("estimate_stream_us", ctypes.c_double)]


def load():
    """Load libfa_b200.so (built in-tree by ``build.build()``); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise ImportError("CUDA library %s is missing; run `python -m paper_2609_21264_b200.build` "
                          "(there is no CPU fallback)" % path)
    lib = ctypes.CDLL(path)
    vp, i32, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.fa_create.restype = i32
    lib.fa_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(fa_config)]
    fwd_args = [vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, f32, vp]
    lib.fa_forward.restype = i32
    lib.fa_forward.argtypes = fwd_args
    lib.fa_forward_host.restype = i32
    lib.fa_forward_host.argtypes = fwd_args
    lib.fa_forward_varlen.restype = i32
    lib.fa_forward_varlen.argtypes = [vp] * 8 + [i32] * 8 + [i32, ctypes.c_float, vp]
    lib.fa_plan.restype = i32
    lib.fa_plan.argtypes = [i32, ctypes.POINTER(fa_config), i32] + [i32] * 8 + [ctypes.POINTER(fa_plan_info)]
    lib.fa_forward_fp8.restype = i32
    lib.fa_forward_fp8.argtypes = [vp] * 9 + [i32] * 7 + [f32, vp]
    lib.fa_forward_mxfp8.restype = i32
    lib.fa_forward_mxfp8.argtypes = [vp] * 9 + [i32] * 7 + [f32, vp]
    lib.fa_forward_strided.restype = i32
    lib.fa_forward_strided.argtypes = fwd_args[:-1] + [vp, vp, vp, vp, vp]
    lib.fa_last_status.restype = i32
    lib.fa_last_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.fa_destroy.restype = i32
    lib.fa_destroy.argtypes = [vp]
    lib.fa_strerror.restype = ctypes.c_char_p
    lib.fa_strerror.argtypes = [i32]
    lib.fa_launch_count.restype = ctypes.c_uint64
    lib.fa_launch_count.argtypes = [vp]
    lib.fa_last_kernel_name.restype = ctypes.c_char_p
    lib.fa_last_kernel_name.argtypes = [vp]
    lib.fa_last_kv_splits.restype = i32
    lib.fa_last_kv_splits.argtypes = [vp]
    lib.fa_forward_split_noalloc.restype = i32
    lib.fa_forward_split_noalloc.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i32, f32, i32, vp]
    lib.fa_noalloc_scratch_bytes.restype = ctypes.c_size_t
    lib.fa_noalloc_scratch_bytes.argtypes = []
    lib.fa_debug_set_drop_v_load.restype = i32
    lib.fa_debug_set_drop_v_load.argtypes = [vp, i32]
    lib.fa_append_paged.restype = i32
    lib.fa_append_paged.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, vp, vp]
    lib.fa_forward_paged.restype = i32
    lib.fa_forward_paged.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, f32, vp, vp, vp]
    lib.fa_forward_paged_diff.restype = i32
    lib.fa_forward_paged_diff.argtypes = [vp, vp, vp, vp, vp, i32, i32, f32, vp, vp, vp, vp]
    lib.fa_forward_diff.restype = i32
    lib.fa_forward_diff.argtypes = [vp] * 5 + [i32] * 8 + [f32] + [vp] * 6
    lib.fa_plan_paged.restype = i32
    lib.fa_plan_paged.argtypes = [i32, vp, vp, vp, i32, i32, i32, vp, vp, i32]
    lib.fa_device.restype = i32
    lib.fa_device.argtypes = [vp]
    lib.fa_noalloc_last_status.restype = i32
    lib.fa_noalloc_last_status.argtypes = [ctypes.POINTER(ctypes.c_uint32)]
    _lib = lib
    return lib


def fa_strerror(status: int) -> str:
    return load().fa_strerror(int(status)).decode()


def fa_create(device: int = -1, flags: int = 0, wait_limit_ms: int = 0, kv_splits: int = 0,
              scratch_bytes: int = 0) -> int:
    """Returns an opaque handle (integer address).  Raises FaError on failure."""
    cfg = fa_config(ctypes.sizeof(fa_config), device, flags, wait_limit_ms, kv_splits, scratch_bytes)
    out = ctypes.c_void_p()
    st = load().fa_create(ctypes.byref(out), ctypes.byref(cfg))
    if st != FA_OK:
        raise FaError(st, "fa_create")
    return out.value


def fa_forward(h, Q, K, V, O, lse, B, Hq, Hkv, Sq, Sk, dqk, dv, causal, scale, stream=0) -> int:
    """Raw call with device pointers as integers; returns the status code."""
    return load().fa_forward(h, Q, K, V, O, lse, B, Hq, Hkv, Sq, Sk, dqk, dv,
                             int(bool(causal)), float(scale), stream)


def fa_forward_strided(h, Q, K, V, O, lse, B, Hq, Hkv, Sq, Sk, dqk, dv, causal, scale,
                       q_strides, k_strides, v_strides, o_strides, stream=0) -> int:
    """Raw call with device pointers and (batch, head, row) strides in elements; returns the status code."""
    arr = [(ctypes.c_int64 * 3)(*[int(x) for x in st]) for st in (q_strides, k_strides, v_strides, o_strides)]
    return load().fa_forward_strided(h, Q, K, V, O, lse, B, Hq, Hkv, Sq, Sk, dqk, dv, int(bool(causal)), float(scale),
                                     arr[0], arr[1], arr[2], arr[3], stream)


def fa_forward_varlen(h, Q, K, V, O, lse, cu_seqlens_q, cu_seqlens_k, B, total_q, total_k, max_sq,
                      Hq, Hkv, dqk, dv, causal, scale, stream=0) -> int:
    """Raw call on packed [total, H, d] device tensors with device int32 offsets; returns the status code."""
    return load().fa_forward_varlen(h, Q, K, V, O, lse, cu_seqlens_q, cu_seqlens_k, B, total_q, total_k, max_sq,
                                    Hq, Hkv, dqk, dv, int(bool(causal)), float(scale), stream)


def fa_forward_fp8(h, Q8, K8, V8, q_scale, k_scale, v_scale, O, lse, B, Hq, Hkv, Sq, Sk, d, causal, scale, stream=0) -> int:
    """Raw call: e4m3 device tensors with block scales (device fp32 arrays or None); returns the status code."""
    return load().fa_forward_fp8(h, Q8, K8, V8, q_scale, k_scale, v_scale, O, lse, B, Hq, Hkv, Sq, Sk, d,
                                 int(bool(causal)), float(scale), stream)


def fa_plan(num_sms, B, Hq, Hkv, Sq, Sk, dqk, dv, causal, *, varlen=False, flags=0, kv_splits=0, scratch_bytes=0) -> dict:
    """What the library would launch for this problem on a device with `num_sms` SMs (no GPU needed)."""
    cfg = fa_config(ctypes.sizeof(fa_config), -1, flags, 0, kv_splits, scratch_bytes)
    out = fa_plan_info()
    st = load().fa_plan(num_sms, ctypes.byref(cfg), int(bool(varlen)), B, Hq, Hkv, Sq, Sk, dqk, dv, int(bool(causal)),
                        ctypes.byref(out))
    if st != FA_OK:
        raise FaError(st, "fa_plan")
    return {"kernel": out.kernel.decode(), "kv_splits": out.kv_splits, "ctas": out.ctas, "heads_per_tile": out.heads_per_tile,
            "estimate_pair_us": out.estimate_pair_us, "estimate_stream_us": out.estimate_stream_us}


def fa_forward_host(h, Q, K, V, O, lse, B, Hq, Hkv, Sq, Sk, dqk, dv, causal, scale, stream=0) -> int:
    """Raw call with HOST pointers as integers; returns the status code."""
    return load().fa_forward_host(h, Q, K, V, O, lse, B, Hq, Hkv, Sq, Sk, dqk, dv,
                                  int(bool(causal)), float(scale), stream)


def fa_last_status(h):
    """(status, detail) of the device-side status word; clears it."""
    detail = ctypes.c_uint32(0)
    st = load().fa_last_status(h, ctypes.byref(detail))
    return st, detail.value


def fa_destroy(h) -> int:
    return load().fa_destroy(h)


def fa_launch_count(h) -> int:
    return int(load().fa_launch_count(h))


def fa_forward_split_noalloc(Q, K, V, O, lse, B, Hq, Hkv, Sq, Sk, dqk, dv, causal, scale, kv_splits, stream=0) -> int:
    """Raw call of the allocation-free split-KV entry point (device pointers as integers, no handle).

    For callers that may not allocate: the split-KV partials live in a fixed 8 MiB array inside
    the library instead of a handle's scratch buffer.  Returns the status code.
    """
    return load().fa_forward_split_noalloc(Q, K, V, O, lse, B, Hq, Hkv, Sq, Sk, dqk, dv,
                                           int(bool(causal)), float(scale), int(kv_splits), stream)


def fa_debug_set_drop_v_load(h, enabled) -> int:
    return int(load().fa_debug_set_drop_v_load(h, int(bool(enabled))))


def fa_noalloc_scratch_bytes() -> int:
    return int(load().fa_noalloc_scratch_bytes())


def fa_noalloc_last_status():
    """(status, wait site) of the allocation-free calls on the current device since the last query; synchronises."""
    detail = ctypes.c_uint32(0)
    st = load().fa_noalloc_last_status(ctypes.byref(detail))
    return int(st), int(detail.value)


def fa_last_kv_splits(h) -> int:
    return int(load().fa_last_kv_splits(h))


def fa_last_kernel_name(h) -> str:
    return load().fa_last_kernel_name(h).decode()


def forward(h, q, k, v, *, causal: bool, scale: float = 0.0, out=None, lse=None, want_lse=True):
    """Attention forward on torch CUDA tensors (bf16, logical shape [B,H,S,d]); returns (O, lse).

    Contiguous tensors go through fa_forward.  Views with other strides (say a [B,S,H,d] buffer
    permuted to [B,H,S,d]) go through fa_forward_strided when their last dimension is contiguous;
    `out`, when not given, then takes q's memory layout.
    """
    import torch
    for t in (q, k, v):
        if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 4:
            raise ValueError("q, k, v must be 4-D bf16 CUDA tensors")
    B, Hq, Sq, dqk = q.shape
    _, Hkv, Sk, dv = v.shape
    dense = all(t.is_contiguous() for t in (q, k, v)) and (out is None or out.is_contiguous())
    if out is None:
        if dense:
            out = torch.empty((B, Hq, Sq, dv), dtype=torch.bfloat16, device=q.device)
        else:   # same dimension order in memory as q
            order = sorted(range(3), key=lambda i: -q.stride(i)) + [3]
            shape = (B, Hq, Sq, dv)
            buf = torch.empty([shape[i] for i in order], dtype=torch.bfloat16, device=q.device)
            out = buf.permute([order.index(i) for i in range(4)])
    if lse is None and want_lse:
        lse = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q.device)
    stream = torch.cuda.current_stream(q.device).cuda_stream
    lse_ptr = lse.data_ptr() if lse is not None else None
    if dense:
        st = fa_forward(h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse_ptr,
                        B, Hq, Hkv, Sq, Sk, dqk, dv, causal, scale, stream)
    else:
        for t in (q, k, v, out):
            if t.stride(3) != 1:
                raise ValueError("the last dimension must be contiguous")
        st = fa_forward_strided(h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse_ptr,
                                B, Hq, Hkv, Sq, Sk, dqk, dv, causal, scale,
                                q.stride()[:3], k.stride()[:3], v.stride()[:3], out.stride()[:3], stream)
    if st != FA_OK:
        raise FaError(st, "fa_forward")
    return out, lse


def forward_varlen(h, q, k, v, cu_seqlens_q, cu_seqlens_k, max_sq: int, *, causal: bool, scale: float = 0.0,
                   want_lse=True):
    """Packed variable-length batch: q [total_q,Hq,d], k/v [total_k,Hkv,d] bf16 CUDA tensors, int32 CUDA
    offset tensors of B+1 entries.  Returns (O [total_q,Hq,dv], lse [Hq,total_q])."""
    import torch
    for t in (q, k, v):
        if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 3:
            raise ValueError("q, k, v must be contiguous 3-D bf16 CUDA tensors")
    for t in (cu_seqlens_q, cu_seqlens_k):
        if t.dtype != torch.int32 or not t.is_cuda or not t.is_contiguous() or t.dim() != 1:
            raise ValueError("cu_seqlens must be contiguous 1-D int32 CUDA tensors")
    total_q, Hq, dqk = q.shape
    total_k, Hkv, dv = v.shape
    B = cu_seqlens_q.numel() - 1
    out = torch.empty((total_q, Hq, dv), dtype=torch.bfloat16, device=q.device)
    lse = torch.empty((Hq, total_q), dtype=torch.float32, device=q.device) if want_lse else None
    st = fa_forward_varlen(h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                           lse.data_ptr() if lse is not None else None,
                           cu_seqlens_q.data_ptr(), cu_seqlens_k.data_ptr(), B, total_q, total_k, int(max_sq),
                           Hq, Hkv, dqk, dv, causal, scale, torch.cuda.current_stream(q.device).cuda_stream)
    if st != FA_OK:
        raise FaError(st, "fa_forward_varlen")
    return out, lse


def forward_fp8(h, q8, k8, v8, q_scale, k_scale, v_scale, *, causal: bool, scale: float = 0.0, want_lse=True):
    """Block-scaled e4m3 attention on torch CUDA tensors: q8/k8/v8 uint8 (or float8_e4m3fn) [B,H,S,d]
    with d = 64 or 128 (or q8/k8 with d = 192 and v8 with 128), scales fp32 CUDA tensors or None.  Returns (O bf16 [B,Hq,Sq,d], lse fp32 [B,Hq,Sq])."""
    import torch
    for t in (q8, k8, v8):
        if t.element_size() != 1 or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError("q8, k8, v8 must be contiguous 4-D one-byte CUDA tensors")
    B, Hq, Sq, d = q8.shape
    _, Hkv, Sk, _ = k8.shape
    dv = 128 if d == 192 else d                 # the 192/128 shapes: V and O have head size 128
    if v8.shape[-1] != dv:
        raise ValueError("v8 must have head size %d" % dv)
    n_qt, n_kt = (Sq + 127) // 128, (Sk + 127) // 128
    for t, shape in ((q_scale, (B, Hq, n_qt)), (k_scale, (B, Hkv, n_kt)), (v_scale, (B, Hkv))):
        if t is not None and (t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous() or tuple(t.shape) != shape):
            raise ValueError("scale tensors must be contiguous fp32 CUDA tensors of shape %s" % (shape,))
    out = torch.empty((B, Hq, Sq, dv), dtype=torch.bfloat16, device=q8.device)
    lse = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q8.device) if want_lse else None
    ptr = lambda t: t.data_ptr() if t is not None else None
    st = fa_forward_fp8(h, q8.data_ptr(), k8.data_ptr(), v8.data_ptr(), ptr(q_scale), ptr(k_scale), ptr(v_scale),
                        out.data_ptr(), ptr(lse), B, Hq, Hkv, Sq, Sk, d, causal, scale,
                        torch.cuda.current_stream(q8.device).cuda_stream)
    if st != FA_OK:
        raise FaError(st, "fa_forward_fp8")
    return out, lse


def fa_forward_mxfp8(h, Q8, K8, V8, q_sf, k_sf, v_sf, O, lse, B, Hq, Hkv, Sq, Sk, d, causal, scale, stream=0) -> int:
    """Raw call of the MX form (e4m3 values, e8m0 scale atoms); device pointers as integers; returns the status code."""
    return load().fa_forward_mxfp8(h, Q8, K8, V8, q_sf, k_sf, v_sf, O, lse, B, Hq, Hkv, Sq, Sk, d,
                                   int(bool(causal)), float(scale), stream)


def forward_mxfp8(h, q8, k8, v8, q_sf, k_sf, v_sf, *, causal: bool, scale: float = 0.0, want_lse=True):
    """MX attention on torch CUDA tensors: q8/k8/v8 uint8 [B,H,S,d] with d = 64 or 128, scale atoms uint8
    [B,H,ceil(S/128),512] in the layout of fa_forward_mxfp8.  Returns (O bf16 [B,Hq,Sq,d], lse fp32 [B,Hq,Sq])."""
    import torch
    for t in (q8, k8, v8, q_sf, k_sf, v_sf):
        if t.element_size() != 1 or not t.is_cuda or not t.is_contiguous() or t.dim() != 4:
            raise ValueError("codes and scale atoms must be contiguous 4-D one-byte CUDA tensors")
    B, Hq, Sq, d = q8.shape
    _, Hkv, Sk, _ = k8.shape
    n_qt, n_kt = (Sq + 127) // 128, (Sk + 127) // 128
    for t, shape in ((q_sf, (B, Hq, n_qt, 512)), (k_sf, (B, Hkv, n_kt, 512)), (v_sf, (B, Hkv, n_kt, 512))):
        if tuple(t.shape) != shape:
            raise ValueError("scale atoms must have shape %s" % (shape,))
    out = torch.empty((B, Hq, Sq, d), dtype=torch.bfloat16, device=q8.device)
    lse = torch.empty((B, Hq, Sq), dtype=torch.float32, device=q8.device) if want_lse else None
    st = fa_forward_mxfp8(h, q8.data_ptr(), k8.data_ptr(), v8.data_ptr(), q_sf.data_ptr(), k_sf.data_ptr(), v_sf.data_ptr(),
                          out.data_ptr(), lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Sq, Sk, d, causal, scale,
                          torch.cuda.current_stream(q8.device).cuda_stream)
    if st != FA_OK:
        raise FaError(st, "fa_forward_mxfp8")
    return out, lse


def fa_device(h) -> int:
    """CUDA device ordinal of the handle (-1 for None)."""
    return int(load().fa_device(h))


def fa_plan_paged(num_sms, seq_lens, Hq, Hkv, Sq, dqk, dv, *, page_size=16, max_pages=0, e4m3=False, diff=False, scratch_bytes=0):
    """How fa_forward_paged deals out a batch with these lengths on a device with `num_sms` SMs (no GPU needed):
    (info dict, list of piece dicts)."""
    lens = (ctypes.c_int32 * len(seq_lens))(*[int(n) for n in seq_lens])
    most = max_pages or max(1, -(-max(seq_lens) // page_size))
    cfg = fa_config(ctypes.sizeof(fa_config), -1, 0, 0, 0, scratch_bytes)
    cache = fa_paged_cache(ctypes.sizeof(fa_paged_cache), FA_CACHE_E4M3 if e4m3 else FA_CACHE_BF16, None, None, 1, page_size, Hkv, dqk, dv)
    seqs = fa_paged_seqs(ctypes.sizeof(fa_paged_seqs), len(seq_lens), None, most, ctypes.addressof(lens), most, 0)
    out, pieces = fa_paged_plan_info(), None
    for n in (0, None):          # how many, then which
        count = int(out.pieces) if n is None else 0
        pieces = (fa_paged_piece * max(1, count))()
        st = load().fa_plan_paged(num_sms, ctypes.addressof(cfg), ctypes.addressof(cache), ctypes.addressof(seqs), Hq, Sq, int(bool(diff)),
                                  ctypes.addressof(out), ctypes.addressof(pieces), count)
        if st != FA_OK:
            raise FaError(st, "fa_plan_paged")
    as_dict = lambda x: {f: getattr(x, f) for f, _ in x._fields_ if f != "reserved"}
    return as_dict(out), [as_dict(x) for x in pieces[:out.pieces]]


def fa_append_paged(h, cache, seqs, cu_seqlens, total, K, V, Q, Q_out, Hq, k_strides, v_strides, q_strides, qo_strides, rope,
                    stream=0) -> int:
    """Raw call: `cache`, `seqs` and `rope` are the structures above (rope may be None), pointers integers, strides
    (token, head) pairs in elements; returns the status code."""
    arr = [None if x is None else _I64x2(*[int(i) for i in x]) for x in (k_strides, v_strides, q_strides, qo_strides)]
    ref = lambda x: None if x is None else ctypes.addressof(x)
    return load().fa_append_paged(h, ref(cache), ref(seqs), cu_seqlens, total, K, V, Q, Q_out, Hq, *arr, ref(rope), stream)


def fa_forward_paged(h, cache, seqs, Q, O, lse, Hq, Sq, scale, q_strides, o_strides, stream=0) -> int:
    """Raw call on a paged cache (structures above, pointers as integers, (token, head) strides); returns the status code."""
    arr = [None if x is None else _I64x2(*[int(i) for i in x]) for x in (q_strides, o_strides)]
    ref = lambda x: None if x is None else ctypes.addressof(x)
    return load().fa_forward_paged(h, ref(cache), ref(seqs), Q, O, lse, Hq, Sq, float(scale), *arr, stream)


def fa_forward_paged_diff(h, cache, seqs, Q, O, Hq, Sq, scale, diff, q_strides, o_strides, stream=0) -> int:
    """Raw call of differential attention on a paged cache; returns the status code."""
    arr = [None if x is None else _I64x2(*[int(i) for i in x]) for x in (q_strides, o_strides)]
    ref = lambda x: None if x is None else ctypes.addressof(x)
    return load().fa_forward_paged_diff(h, ref(cache), ref(seqs), Q, O, Hq, Sq, float(scale), ref(diff), *arr, stream)


def fa_forward_diff(h, Q, K, V, O, B, Hq, Hkv, Sq, Sk, dqk, dv, causal, scale, diff, q_strides, k_strides, v_strides, o_strides,
                    stream=0) -> int:
    """Raw call of differential attention on dense tensors with (batch, head, row) strides; returns the status code."""
    arr = [None if x is None else _I64x3(*[int(i) for i in x]) for x in (q_strides, k_strides, v_strides, o_strides)]
    return load().fa_forward_diff(h, Q, K, V, O, B, Hq, Hkv, Sq, Sk, dqk, dv, int(bool(causal)), float(scale),
                                  None if diff is None else ctypes.addressof(diff), *arr, stream)


class PagedCache:
    """A paged key/value cache for the paged entry points.

    k [num_pages, Hkv, page_size, dqk] and v [num_pages, Hkv, page_size, dv]: CUDA tensors of that logical shape in any order of
    the first three dimensions in memory (a [pages, page_size, Hkv, d] pool is passed permuted), bf16, or e4m3
    (torch.float8_e4m3fn or uint8 codes) with one fp32 scale per K/V head.  Make it once per cache; it keeps the tensors alive.
    """

    def __init__(self, k, v, k_scale=None, v_scale=None):
        import torch
        if k.dim() != 4 or v.dim() != 4 or k.shape[:3] != v.shape[:3] or k.dtype != v.dtype:
            raise ValueError("k and v must be 4-D tensors of one dtype with the same pages, heads and page size")
        if k.dtype not in (torch.bfloat16, torch.float8_e4m3fn, torch.uint8):
            raise ValueError("the cache must be bf16 or e4m3")
        if not k.is_cuda or v.device != k.device or k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("k and v must be on one CUDA device, their last dimension contiguous")
        for t in (k_scale, v_scale):
            if t is not None and (t.dtype != torch.float32 or t.device != k.device or not t.is_contiguous() or
                                  tuple(t.shape) != (k.shape[1],) or k.dtype == torch.bfloat16):
                raise ValueError("scales are contiguous fp32 tensors of Hkv values on the cache's device, for e4m3 caches only")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        load()                            # the calls that take a cache rely on the library being there
        self.device, self.Hkv, self.dqk, self.dv = k.device, k.shape[1], k.shape[3], v.shape[3]
        # (a single page or head may have any stride, the library wants a valid one: whole 16-byte units)
        unit = 16 // k.element_size()
        strides = [_I64x3(*[s if n > 1 else max(t.shape[3], -(-s // unit) * unit) for s, n in zip(t.stride(), t.shape[:3])]) for t in (k, v)]
        self.c = fa_paged_cache(ctypes.sizeof(fa_paged_cache), FA_CACHE_BF16 if k.dtype == torch.bfloat16 else FA_CACHE_E4M3,
                                k.data_ptr(), v.data_ptr(), k.shape[0], k.shape[2], k.shape[1], k.shape[3], v.shape[3], 0,
                                *strides,
                                None if k_scale is None else k_scale.data_ptr(), None if v_scale is None else v_scale.data_ptr())
        self.address = ctypes.addressof(self.c)


class Rope:
    """Rotation by position for `append_paged`: cos_sin is a contiguous fp32 CUDA tensor [max_pos, dim] (dim/2 cosines, then
    dim/2 sines per position); of every `span` dimensions of a head (0: the whole head) those from `offset` on are turned, as
    halves or in interleaved pairs."""

    def __init__(self, cos_sin, *, offset: int = 0, span: int = 0, interleaved: bool = False):
        import torch
        if cos_sin.dtype != torch.float32 or not cos_sin.is_cuda or not cos_sin.is_contiguous() or cos_sin.dim() != 2:
            raise ValueError("cos_sin must be a contiguous 2-D fp32 CUDA tensor")
        self.cos_sin, self.device, self.span = cos_sin, cos_sin.device, int(span)
        self.offset, self.interleaved = int(offset), int(bool(interleaved))
        self.structs = {}                 # by span

    def struct_for(self, dqk: int) -> int:
        """Address of the C structure for heads of dqk dimensions."""
        span = self.span or dqk
        c = self.structs.get(span)
        if c is None:
            t = self.cos_sin
            c = self.structs[span] = fa_rope(ctypes.sizeof(fa_rope), t.shape[0], t.data_ptr(), t.shape[1], self.offset, span, self.interleaved)
        return ctypes.addressof(c)


# The calls below are made once per layer and token: their checks are written to cost little (one stride array per call, the raw
# stream, attributes read once).

def _raw_stream(device) -> int:
    """The current stream's handle on `device` (torch.cuda.current_stream without the object around it)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(device.index)


def _seqs(h, cache, block_table, seq_lens):
    """The fa_paged_seqs of a call, after the checks that all paged calls share."""
    import torch
    i32, device = torch.int32, cache.device
    if block_table.dtype is not i32 or block_table.device != device or block_table.dim() != 2:
        raise ValueError("block_table must be a 2-D int32 tensor on the cache's device")
    B, max_pages = block_table.shape
    stride, inner = block_table.stride()
    if (inner != 1 and max_pages > 1) or (stride < max_pages and B > 1):
        raise ValueError("the rows of block_table must be contiguous and lie apart")
    if seq_lens.dtype is not i32 or seq_lens.device != device or seq_lens.shape != (B,) or not seq_lens.is_contiguous():
        raise ValueError("seq_lens must be a contiguous int32 tensor of one length per row of block_table")
    if _lib.fa_device(h) != device.index:
        raise ValueError("the handle belongs to another device than the cache")
    # (the stride of a single row is whatever the view left)
    return fa_paged_seqs(_SEQS_SIZE, B, block_table.data_ptr(), stride if B > 1 else max_pages, seq_lens.data_ptr(),
                         max_pages, 0)


def _rows(t, cache, d, what):
    """Tokens, heads and (token, head) strides of a [tokens, heads, d] bf16 tensor on the cache's device."""
    import torch
    if t.dtype is not torch.bfloat16 or t.device != cache.device or t.dim() != 3:
        raise ValueError("%s must be a 3-D bf16 tensor on the cache's device" % what)
    n, heads, width = t.shape
    st, sh, sd = t.stride()
    if width != d or sd != 1:
        raise ValueError("the last dimension of %s must be %d contiguous values" % (what, d))
    # (the stride of a dimension of one row is whatever the view left; the library wants it to be valid)
    if n <= 1:
        st = max(d, (st + 7) // 8 * 8)
    if heads == 1:
        sh = max(d, (sh + 7) // 8 * 8)
    return n, heads, st, sh


def _new(q, tokens, heads, d):
    """A contiguous [tokens, heads, d] tensor of q's type (the cheapest way to it)."""
    import torch
    return torch.empty_like(q) if q.shape[2] == d and q.is_contiguous() else q.new_empty((tokens, heads, d))


def append_paged(h, k, v, cache: PagedCache, block_table, seq_lens, *, cu_seqlens=None, q=None, q_out=None, rope: Rope = None):
    """New keys and values [T, Hkv, d] of packed tokens into `cache`, rotated by their positions; returns q_out.

    seq_lens [B] int32 counts the new tokens in; cu_seqlens [B+1] int32 gives each sequence's rows (None: T / B each).  With q
    [T, Hq, dqk] the queries are rotated too, into q_out (allocated when not given; may be q itself).
    """
    import torch
    seqs = _seqs(h, cache, block_table, seq_lens)
    total, Hk, kt, kh = _rows(k, cache, cache.dqk, "k")
    Tv, Hv, vt, vh = _rows(v, cache, cache.dv, "v")
    if Tv != total or Hk != cache.Hkv or Hv != Hk:
        raise ValueError("k and v must have the same tokens and the cache's heads")
    cu_ptr = None
    if cu_seqlens is not None:
        if (cu_seqlens.dtype is not torch.int32 or cu_seqlens.device != cache.device or cu_seqlens.shape != (seqs.B + 1,) or
                not cu_seqlens.is_contiguous()):
            raise ValueError("cu_seqlens must be a contiguous int32 tensor of B + 1 offsets on the cache's device")
        cu_ptr = cu_seqlens.data_ptr()
    rope_ptr = None
    if rope is not None:
        if rope.device != cache.device:
            raise ValueError("the rotation table must be on the cache's device")
        rope_ptr = rope.struct_for(cache.dqk)
    q_ptr = qo_ptr = None
    Hq = qt = qh = ot = oh = 0
    if q is not None:
        Tq, Hq, qt, qh = _rows(q, cache, cache.dqk, "q")
        if Tq != total:
            raise ValueError("q must have the tokens of k")
        if q_out is None:
            q_out = _new(q, total, Hq, cache.dqk)
            ot, oh = Hq * cache.dqk, cache.dqk
        else:
            To, Ho, ot, oh = _rows(q_out, cache, cache.dqk, "q_out")
            if To != total or Ho != Hq:
                raise ValueError("q_out must have q's shape")
        q_ptr, qo_ptr = q.data_ptr(), q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    strides = _I64x8(kt, kh, vt, vh, qt, qh, ot, oh)
    at = ctypes.addressof(strides)
    st = _lib.fa_append_paged(h, cache.address, ctypes.addressof(seqs), cu_ptr, total, k.data_ptr(), v.data_ptr(), q_ptr, qo_ptr, Hq,
                              at, at + 16, at + 32, at + 48, rope_ptr, _raw_stream(cache.device))
    if st != FA_OK:
        raise FaError(st, "fa_append_paged")
    return q_out


def _paged_out(q, cache, seqs, out):
    """(Hq, tokens, Sq, stride array, out) of a paged attention call."""
    import torch
    T, Hq, qt, qh = _rows(q, cache, cache.dqk, "q")
    B = seqs.B
    if T != 0 if B == 0 else T == 0 or T % B:
        raise ValueError("q must hold the same number of tokens for every sequence")
    if out is None:
        out = _new(q, T, Hq, cache.dv)
        ot, oh = Hq * cache.dv, cache.dv
    else:
        To, Ho, ot, oh = _rows(out, cache, cache.dv, "out")
        if To != T or Ho != Hq:
            raise ValueError("out must have shape %s" % ((T, Hq, cache.dv),))
    return Hq, T, T // B if B else 1, _I64x4(qt, qh, ot, oh), out


def forward_paged(h, q, cache: PagedCache, block_table, seq_lens, *, scale: float = 0.0, out=None, want_lse=True):
    """Attention of the last tokens of every sequence over a paged cache: q [B*Sq, Hq, dqk] bf16; returns (O [B*Sq, Hq, dv],
    lse [Hq, B*Sq] fp32 or None).  A batch of no sequences launches nothing."""
    import torch
    seqs = _seqs(h, cache, block_table, seq_lens)
    Hq, T, Sq, strides, out = _paged_out(q, cache, seqs, out)
    lse = q.new_empty((Hq, T), dtype=torch.float32) if want_lse else None
    at = ctypes.addressof(strides)
    st = _lib.fa_forward_paged(h, cache.address, ctypes.addressof(seqs), q.data_ptr(), out.data_ptr(),
                               None if lse is None else lse.data_ptr(), Hq, Sq, scale, at, at + 16, _raw_stream(cache.device))
    if st != FA_OK:
        raise FaError(st, "fa_forward_paged")
    return out, lse


def _diff(lam, norm_weight, eps, out_scale, Hq, device):
    import torch
    if lam.dtype != torch.float32 or lam.device != device or tuple(lam.shape) != (Hq,) or not lam.is_contiguous():
        raise ValueError("lam must be a contiguous fp32 tensor of one value per query head")
    if norm_weight is not None and (norm_weight.dtype != torch.float32 or norm_weight.device != device or
                                    tuple(norm_weight.shape) != (128,) or not norm_weight.is_contiguous()):
        raise ValueError("norm_weight must be a contiguous fp32 tensor of 128 values")
    return fa_diff(ctypes.sizeof(fa_diff), eps, lam.data_ptr(), None if norm_weight is None else norm_weight.data_ptr(), out_scale, 0.0)


def forward_paged_diff(h, q, cache: PagedCache, block_table, seq_lens, lam, *, norm_weight=None, eps: float = 1e-5,
                       out_scale: float = 1.0, scale: float = 0.0, out=None):
    """Differential attention of the last tokens over a paged cache whose heads are two maps of 64 and values of 128; returns O."""
    seqs = _seqs(h, cache, block_table, seq_lens)
    Hq, T, Sq, strides, out = _paged_out(q, cache, seqs, out)
    diff = _diff(lam, norm_weight, eps, out_scale, Hq, cache.device)
    at = ctypes.addressof(strides)
    st = _lib.fa_forward_paged_diff(h, cache.address, ctypes.addressof(seqs), q.data_ptr(), out.data_ptr(), Hq, Sq, scale,
                                    ctypes.addressof(diff), at, at + 16, _raw_stream(cache.device))
    if st != FA_OK:
        raise FaError(st, "fa_forward_paged_diff")
    return out


def forward_diff(h, q, k, v, lam, *, causal: bool, norm_weight=None, eps: float = 1e-5, out_scale: float = 1.0, scale: float = 0.0,
                 out=None):
    """Differential attention on torch CUDA tensors (bf16, logical shape [B, H, S, 128], any batch/head/row strides; the two
    halves of a query and key are its two maps); returns O, in q's memory layout when `out` is not given."""
    import torch
    lib, device, bf16 = load(), q.device, torch.bfloat16
    if not q.is_cuda or any(t.dtype is not bf16 or t.dim() != 4 or t.device != device for t in (q, k, v)):
        raise ValueError("q, k, v must be 4-D bf16 tensors on one CUDA device")
    B, Hq, Sq, dqk = q.shape
    _, Hkv, Sk, dv = v.shape
    if k.shape != (B, Hkv, Sk, dqk) or v.shape[0] != B:
        raise ValueError("k and v must have q's batch, the same heads and rows, and k q's head size")
    if lib.fa_device(h) != device.index:
        raise ValueError("the handle belongs to another device than the tensors")
    shape = (B, Hq, Sq, dv)
    if out is None:
        if q.is_contiguous():
            out = torch.empty(shape, dtype=bf16, device=device)
        else:
            order = sorted(range(3), key=lambda i: -q.stride(i)) + [3]
            buf = torch.empty([shape[i] for i in order], dtype=bf16, device=device)
            out = buf.permute([order.index(i) for i in range(4)])
    elif out.shape != shape or out.dtype is not bf16 or out.device != device:
        raise ValueError("out must be a bf16 tensor of shape %s on q's device" % (shape,))
    strides = []
    for t in (q, k, v, out):
        s = t.stride()
        if s[3] != 1:
            raise ValueError("the last dimension must be contiguous")
        # (a dimension of one entry may have any stride, the library wants a valid one; a row holds 128 values)
        strides += s[:3] if min(t.shape) > 1 else [x if n > 1 else max(128, (x + 7) // 8 * 8) for x, n in zip(s[:3], t.shape)]
    strides = _I64x12(*strides)
    at = ctypes.addressof(strides)
    diff = _diff(lam, norm_weight, eps, out_scale, Hq, device)
    st = lib.fa_forward_diff(h, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, Hq, Hkv, Sq, Sk, dqk, dv, 1 if causal else 0,
                             scale, ctypes.addressof(diff), at, at + 24, at + 48, at + 72, _raw_stream(device))
    if st != FA_OK:
        raise FaError(st, "fa_forward_diff")
    return out
