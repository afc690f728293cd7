"""Thin Python front end of the C-ABI library (include/hyd_attn.h): argument marshalling only.
PyTorch supplies device memory and the current HIP stream; every step of the computation runs in
the library's HIP kernels.  There is no fallback: if the library is missing or a call fails, an
exception is raised."""
import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libhyd_attn.so")
HYD_BF16, HYD_FP32 = 0, 1
_lib = None

EXPORTS = (
    "hyd_status_string", "hyd_varlen_attn_workspace_bytes", "hyd_varlen_attn_fwd",
    "hyd_varlen_attn_bwd", "hyd_enable_kernel_timing", "hyd_kernel_times", "hyd_set_wg_trace",
    "hyd_varlen_attn_fwd_range", "hyd_varlen_attn_bwd_range", "hyd_attn_merge", "hyd_rope_packed",
    "hyd_varlen_attn_fwd_noalloc", "hyd_varlen_attn_fwd_noalloc_max_workspace",
    "hyd_varlen_attn_schedule_status", "hyd_varlen_attn_schedule_layout",
    "hyd_varlen_attn_fwd_rope", "hyd_varlen_attn_bwd_rope", "hyd_rope_rotate", "hyd_rope_frequencies",
    "hyd_cross_attn_workspace_bytes", "hyd_cross_attn_fwd", "hyd_cross_attn_bwd",
)
RANGE_ALIGN = 256   # HYD_RANGE_ALIGN of the header
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}                  # hyd_rope_layout
ROPE_SCALINGS = {"plain": 0, "linear": 1, "parts": 2}         # hyd_rope_scaling


class HydError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"hyd_attn error {code}: {msg}")
        self.code = code


def load():
    """Load libhyd_attn.so (built by paper_2412_07894_amd/build.py; never built implicitly here)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python paper_2412_07894_amd/build.py` "
            "(or __graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, ip, i, f, sz = ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    lib.hyd_status_string.restype = ctypes.c_char_p
    lib.hyd_status_string.argtypes = [i]
    lib.hyd_varlen_attn_workspace_bytes.restype = sz
    lib.hyd_varlen_attn_workspace_bytes.argtypes = [i, i, i, i, i, i, i]
    lib.hyd_varlen_attn_fwd.restype = i
    lib.hyd_varlen_attn_fwd.argtypes = [vp, vp, vp, ip, i, ip, i, i, i, i, i, f, i, vp, vp, vp, sz, vp]
    lib.hyd_varlen_attn_fwd_noalloc.restype = i
    lib.hyd_varlen_attn_fwd_noalloc.argtypes = [vp, vp, vp, ip, i, ip, i, i, i, i, i, f, i, vp, vp, vp]
    lib.hyd_varlen_attn_fwd_noalloc_max_workspace.restype = sz
    lib.hyd_varlen_attn_fwd_noalloc_max_workspace.argtypes = []
    lib.hyd_varlen_attn_schedule_status.restype = i
    lib.hyd_varlen_attn_schedule_status.argtypes = [vp, sz, i, i, i, i, i, i, i, vp]
    lib.hyd_varlen_attn_schedule_layout.restype = i
    lib.hyd_varlen_attn_schedule_layout.argtypes = [i, i, i, i, i, i, i, i, ctypes.POINTER(sz), ctypes.POINTER(sz),
                                                    ctypes.POINTER(i), ctypes.POINTER(i)]
    lib.hyd_varlen_attn_fwd_rope.restype = i
    lib.hyd_varlen_attn_fwd_rope.argtypes = [vp, vp, vp, ip, i, ip, i, i, i, i, i, f, f, i, vp, vp, vp, sz, vp]
    lib.hyd_varlen_attn_bwd_rope.restype = i
    lib.hyd_varlen_attn_bwd_rope.argtypes = [vp, vp, vp, vp, vp, vp, ip, i, ip, i, i, i, i, i, f, f, i,
                                             vp, vp, vp, vp, sz, vp]
    lib.hyd_varlen_attn_bwd.restype = i
    lib.hyd_varlen_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, ip, i, ip, i, i, i, i, i, f, i,
                                        vp, vp, vp, vp, sz, vp]
    lib.hyd_varlen_attn_fwd_range.restype = i
    lib.hyd_varlen_attn_fwd_range.argtypes = [vp, vp, vp, ip, i, ip, ip, ip, i, i, i, i, i, f, i, vp, vp, vp, sz, vp]
    lib.hyd_varlen_attn_bwd_range.restype = i
    lib.hyd_varlen_attn_bwd_range.argtypes = [vp, vp, vp, vp, vp, vp, ip, i, ip, ip, ip, i, i, i, i, i, f, i,
                                              vp, vp, vp, vp, sz, vp]
    lib.hyd_attn_merge.restype = i
    lib.hyd_attn_merge.argtypes = [vp, vp, vp, vp, i, i, i, i, vp, vp, vp]
    lib.hyd_rope_packed.restype = i
    lib.hyd_rope_packed.argtypes = [vp, ip, i, i, i, i, f, i, i, vp, vp]
    lib.hyd_cross_attn_workspace_bytes.restype = sz
    lib.hyd_cross_attn_workspace_bytes.argtypes = [i] * 10
    lib.hyd_cross_attn_fwd.restype = i
    lib.hyd_cross_attn_fwd.argtypes = [vp, vp, vp, ip, ip, ip, i, ip, ip, i, i, i, i, i, i, i, f, i, vp, vp, vp, sz, vp]
    lib.hyd_cross_attn_bwd.restype = i
    lib.hyd_cross_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, ip, ip, ip, i, ip, ip, i, i, i, i, i, i, i, f, i, vp, vp, vp, vp, sz, vp]
    l, dbl = ctypes.c_int64, ctypes.c_double
    lib.hyd_rope_rotate.restype = i
    lib.hyd_rope_rotate.argtypes = [vp, i, l, vp, l, vp, i, l, vp, l, ip, ip, i, ip, i, i, vp, i, i, f, i, i, vp]
    lib.hyd_rope_frequencies.restype = i
    lib.hyd_rope_frequencies.argtypes = [i, dbl, i, dbl, dbl, dbl, dbl, vp]
    lib.hyd_enable_kernel_timing.restype = None
    lib.hyd_enable_kernel_timing.argtypes = [i]
    lib.hyd_kernel_times.restype = i
    lib.hyd_kernel_times.argtypes = [ctypes.POINTER(ctypes.c_char_p), ctypes.POINTER(ctypes.c_float), i]
    lib.hyd_set_wg_trace.restype = None
    lib.hyd_set_wg_trace.argtypes = [vp, i]
    _lib = lib
    return lib


def status_string(code):
    return load().hyd_status_string(int(code)).decode()


def _check(code):
    if code != 0:
        raise HydError(code, status_string(code))


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return HYD_BF16
    if t.dtype == torch.float32:
        return HYD_FP32
    raise TypeError(f"unsupported dtype {t.dtype}")


def workspace_bytes(total_tokens, num_seqs, hq, hkv, head_dim, dtype_code, is_bwd):
    return int(load().hyd_varlen_attn_workspace_bytes(total_tokens, num_seqs, hq, hkv, head_dim,
                                                      dtype_code, int(is_bwd)))


def _workspace(nbytes, device):
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def _host_ptr(cu_host):
    if cu_host is None:
        return None, None
    keep = (ctypes.c_int32 * len(cu_host))(*[int(x) for x in cu_host])
    return keep, ctypes.cast(keep, ctypes.c_void_p)


def _stream_ptr(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _on_device(device, call, args, stream):
    """call(*args, stream) with the device of the call's tensors as the current one, on `stream` or else that device's current one.
    (Small calls take as long as the host does: the stream's handle and the device are asked for without an object around them.)"""
    if device.type != "cuda":
        raise ValueError(f"tensors must be on a GPU, got {device}")
    index = device.index
    handle = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream
    if index == torch._C._cuda_getDevice():
        code = call(*args, handle)
    else:
        with torch.cuda.device(index):
            code = call(*args, handle)
    if code != 0:
        raise HydError(code, status_string(code))


def varlen_attn_fwd(q, k, v, cu_seqlens, max_seqlen, softmax_scale, cu_seqlens_host=None,
                    workspace=None, stream=None, out=None, lse=None, rope_base=None):
    """q[T,Hq,d], k,v[T,Hkv,d] contiguous device tensors (bf16 or fp32); cu_seqlens int32 device
    tensor [num_seqs+1].  Returns (o[T,Hq,d], lse[Hq,T] fp32).  With rope_base the call is
    hyd_varlen_attn_fwd_rope: q unrotated (rotated inside the kernel), k already rotated."""
    lib = load()
    T, hq, d = q.shape
    hkv = k.shape[1]
    assert q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
    assert cu_seqlens.dtype == torch.int32 and cu_seqlens.is_contiguous()
    dt = _dtype_code(q)
    nseq = cu_seqlens.numel() - 1
    o = torch.empty_like(q) if out is None else out
    lse = torch.empty((hq, T), dtype=torch.float32, device=q.device) if lse is None else lse
    need = workspace_bytes(T, nseq, hq, hkv, d, dt, False)
    ws = _workspace(need, q.device) if workspace is None else workspace
    keep, hp = _host_ptr(cu_seqlens_host)
    if rope_base is None:
        _check(lib.hyd_varlen_attn_fwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(), nseq,
                                       hp, T, int(max_seqlen), hq, hkv, d, float(softmax_scale), dt,
                                       o.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(),
                                       _stream_ptr(stream)))
    else:
        _check(lib.hyd_varlen_attn_fwd_rope(q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(), nseq,
                                            hp, T, int(max_seqlen), hq, hkv, d, float(softmax_scale), float(rope_base), dt,
                                            o.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel(),
                                            _stream_ptr(stream)))
    return o, lse


def varlen_attn_fwd_noalloc(q, k, v, cu_seqlens, max_seqlen, softmax_scale, out, lse, cu_seqlens_host=None, stream=None):
    """The forward without a workspace: the library keeps the schedule in an array of its own
    (see the header); `out` and `lse` are caller-owned, nothing is allocated here or there."""
    T, hq, d = q.shape
    hkv = k.shape[1]
    for t in (q, k, v, out, lse, cu_seqlens):
        assert t.is_contiguous()
    assert out.shape == q.shape and out.dtype == q.dtype and lse.dtype == torch.float32 and lse.shape == (hq, T)
    keep, hp = _host_ptr(cu_seqlens_host)
    _check(load().hyd_varlen_attn_fwd_noalloc(q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(),
                                              cu_seqlens.numel() - 1, hp, T, int(max_seqlen), hq, hkv, d,
                                              float(softmax_scale), _dtype_code(q), out.data_ptr(), lse.data_ptr(),
                                              _stream_ptr(stream)))
    return out, lse


def varlen_attn_bwd(q, k, v, o, lse, d_o, cu_seqlens, max_seqlen, softmax_scale, cu_seqlens_host=None,
                    workspace=None, stream=None, dq=None, dk=None, dv=None, rope_base=None):
    """Returns (dq, dk, dv) with the shapes and dtype of q, k, v.  With rope_base the call is
    hyd_varlen_attn_bwd_rope: q unrotated, k rotated; dq is for the unrotated q, dk for the rotated k."""
    lib = load()
    T, hq, d = q.shape
    hkv = k.shape[1]
    for t in (q, k, v, o, d_o, lse):
        assert t.is_contiguous()
    dt = _dtype_code(q)
    nseq = cu_seqlens.numel() - 1
    dq = torch.empty_like(q) if dq is None else dq
    dk = torch.empty_like(k) if dk is None else dk
    dv = torch.empty_like(v) if dv is None else dv
    need = workspace_bytes(T, nseq, hq, hkv, d, dt, True)
    ws = _workspace(need, q.device) if workspace is None else workspace
    keep, hp = _host_ptr(cu_seqlens_host)
    if rope_base is None:
        _check(lib.hyd_varlen_attn_bwd(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                                       d_o.data_ptr(), cu_seqlens.data_ptr(), nseq, hp, T, int(max_seqlen),
                                       hq, hkv, d, float(softmax_scale), dt, dq.data_ptr(), dk.data_ptr(),
                                       dv.data_ptr(), ws.data_ptr(), ws.numel(), _stream_ptr(stream)))
    else:
        _check(lib.hyd_varlen_attn_bwd_rope(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                                            d_o.data_ptr(), cu_seqlens.data_ptr(), nseq, hp, T, int(max_seqlen),
                                            hq, hkv, d, float(softmax_scale), float(rope_base), dt, dq.data_ptr(),
                                            dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), ws.numel(), _stream_ptr(stream)))
    return dq, dk, dv


def _ranges_args(ranges, nseq, device):
    """ranges: sequence of (q_begin, q_end, kv_begin, kv_end) per sequence -> (device tensor, host
    array kept alive, host pointer)."""
    flat = [int(x) for r in ranges for x in r]
    assert len(flat) == 4 * nseq, "one (q_begin, q_end, kv_begin, kv_end) per sequence"
    dev = torch.tensor(flat, dtype=torch.int32, device=device) if nseq else torch.zeros(4, dtype=torch.int32, device=device)
    keep = (ctypes.c_int32 * max(len(flat), 1))(*flat)
    return dev, keep, ctypes.cast(keep, ctypes.c_void_p)


def varlen_attn_fwd_range(q, k, v, cu_seqlens, ranges, max_seqlen, softmax_scale, out, lse,
                          cu_seqlens_host=None, workspace=None, stream=None):
    """One visit of a key range to a query range for every sequence (see the header).  `out` and
    `lse` are caller-owned and only the rows of the query ranges are written."""
    lib = load()
    T, hq, d = q.shape
    hkv = k.shape[1]
    for t in (q, k, v, out, lse, cu_seqlens):
        assert t.is_contiguous()
    assert lse.dtype == torch.float32 and lse.shape == (hq, T) and out.shape == q.shape and out.dtype == q.dtype
    dt = _dtype_code(q)
    nseq = cu_seqlens.numel() - 1
    need = workspace_bytes(T, nseq, hq, hkv, d, dt, False)
    ws = _workspace(need, q.device) if workspace is None else workspace
    keep, hp = _host_ptr(cu_seqlens_host)
    rdev, rkeep, rhp = _ranges_args(ranges, nseq, q.device)
    _check(lib.hyd_varlen_attn_fwd_range(q.data_ptr(), k.data_ptr(), v.data_ptr(), cu_seqlens.data_ptr(), nseq,
                                         hp, rdev.data_ptr(), rhp, T, int(max_seqlen), hq, hkv, d,
                                         float(softmax_scale), dt, out.data_ptr(), lse.data_ptr(),
                                         ws.data_ptr(), ws.numel(), _stream_ptr(stream)))
    return out, lse


def varlen_attn_bwd_range(q, k, v, o, lse, d_o, cu_seqlens, ranges, max_seqlen, softmax_scale, dq, dk, dv,
                          cu_seqlens_host=None, workspace=None, stream=None):
    """Partial gradients of one visit; o and lse are the merged forward results.  dq / dk / dv are
    caller-owned; only the rows of the query (dq) and key (dk, dv) ranges are written."""
    lib = load()
    T, hq, d = q.shape
    hkv = k.shape[1]
    for t in (q, k, v, o, d_o, lse, dq, dk, dv, cu_seqlens):
        assert t.is_contiguous()
    assert dq.shape == q.shape and dk.shape == k.shape and dv.shape == v.shape
    dt = _dtype_code(q)
    nseq = cu_seqlens.numel() - 1
    need = workspace_bytes(T, nseq, hq, hkv, d, dt, True)
    ws = _workspace(need, q.device) if workspace is None else workspace
    keep, hp = _host_ptr(cu_seqlens_host)
    rdev, rkeep, rhp = _ranges_args(ranges, nseq, q.device)
    _check(lib.hyd_varlen_attn_bwd_range(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(),
                                         d_o.data_ptr(), cu_seqlens.data_ptr(), nseq, hp, rdev.data_ptr(), rhp,
                                         T, int(max_seqlen), hq, hkv, d, float(softmax_scale), dt,
                                         dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), ws.numel(),
                                         _stream_ptr(stream)))
    return dq, dk, dv


def attn_merge(o_a, lse_a, o_b, lse_b, out=None, lse_out=None, stream=None):
    """Log-sum-exp merge of two partial results; out / lse_out may be either input pair."""
    T, hq, d = o_a.shape
    out = torch.empty_like(o_a) if out is None else out
    lse_out = torch.empty_like(lse_a) if lse_out is None else lse_out
    for t in (o_a, lse_a, o_b, lse_b, out, lse_out):
        assert t.is_contiguous()
    assert o_b.shape == o_a.shape and lse_a.shape == (hq, T) and lse_b.shape == (hq, T)
    _check(load().hyd_attn_merge(o_a.data_ptr(), lse_a.data_ptr(), o_b.data_ptr(), lse_b.data_ptr(), T, hq, d,
                                 _dtype_code(o_a), out.data_ptr(), lse_out.data_ptr(), _stream_ptr(stream)))
    return out, lse_out


def rope_packed(x, cu_seqlens, base=10000.0, inverse=False, out=None, stream=None):
    """Rotary embedding with per-sequence position reset on x[T,H,d] (bf16); out may be x."""
    T, h, d = x.shape
    out = torch.empty_like(x) if out is None else out
    assert x.is_contiguous() and out.is_contiguous() and out.shape == x.shape and out.dtype == x.dtype
    assert cu_seqlens.dtype == torch.int32 and cu_seqlens.is_contiguous()
    _check(load().hyd_rope_packed(x.data_ptr(), cu_seqlens.data_ptr(), cu_seqlens.numel() - 1, T, h, d, float(base),
                                  int(bool(inverse)), _dtype_code(x), out.data_ptr(), _stream_ptr(stream)))
    return out


def cross_attn_workspace_bytes(total_q, total_kv, num_seqs, max_seqlen_q, max_seqlen_kv, hq, hkv, head_dim, dtype_code, is_bwd):
    """Bytes of workspace of cross_attn_fwd (is_bwd false) or cross_attn_bwd; 0 for sizes that are refused."""
    return int(load().hyd_cross_attn_workspace_bytes(total_q, total_kv, num_seqs, max_seqlen_q, max_seqlen_kv, hq, hkv, head_dim,
                                                     dtype_code, int(bool(is_bwd))))


def _made(shape, dtype, device, stream):
    """A new tensor that belongs to the stream its kernel runs on: its memory may have been another tensor's of that stream, but of no
    other stream that still works on it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _like(name, t, shape, dtype, device, stream=None):
    """t as it is, checked; made for `stream` if None."""
    if t is None:
        return _made(shape, dtype, device, stream)
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {tuple(shape)} tensor of {dtype} on {device}, got {tuple(t.shape)} {t.dtype} {t.device}")
    return t


def _cross_sizes(q, k, v, cu_q, cu_kv, max_seqlen_q, max_seqlen_kv, workspace, is_bwd, stream):
    """Checks of the tensors that both directions take: (Tq, Tk, num_seqs, Hq, Hkv, d, dtype code, workspace)."""
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError(f"q and k must be [rows, heads, d], got {tuple(q.shape)} and {tuple(k.shape)}")
    (Tq, hq, d), (Tk, hkv, _), dev = q.shape, k.shape, q.device
    dt = _dtype_code(q)
    if not q.is_contiguous():
        raise ValueError(f"q must be contiguous, got strides {q.stride()}")
    _like("k", k, (Tk, hkv, d), q.dtype, dev)
    _like("v", v, (Tk, hkv, d), q.dtype, dev)
    nseq = cu_q.numel() - 1
    if nseq < 0 or cu_kv.numel() != nseq + 1:
        raise ValueError(f"cu_q and cu_kv must have num_seqs + 1 elements, got {cu_q.numel()} and {cu_kv.numel()}")
    if workspace is None:
        nbytes = cross_attn_workspace_bytes(Tq, Tk, nseq, max_seqlen_q, max_seqlen_kv, hq, hkv, d, dt, is_bwd)
        workspace = _made(max(nbytes, 256), torch.uint8, dev, stream)
    elif workspace.dtype != torch.uint8 or not workspace.is_contiguous() or workspace.device != dev:
        raise ValueError(f"workspace must be a contiguous uint8 tensor on {dev}, got {workspace.dtype} {workspace.device}")
    return Tq, Tk, nseq, hq, hkv, d, dt, workspace


def _host_lens(name, cu_host, nseq):
    if cu_host is not None and len(cu_host) != nseq + 1:
        raise ValueError(f"{name} must have num_seqs + 1 = {nseq + 1} elements, got {len(cu_host)}")
    return _host_ptr(cu_host)


def cross_attn_fwd(q, k, v, cu_q, cu_kv, max_seqlen_q, max_seqlen_kv, softmax_scale, kv_lens=None, cu_q_host=None, cu_kv_host=None,
                   workspace=None, stream=None, out=None, lse=None):
    """Cross attention of packed batches: queries q[Tq,Hq,d] of sequence s (rows cu_q[s]..cu_q[s+1]) on all its keys in k, v[Tk,Hkv,d]
    (rows cu_kv[s]..cu_kv[s+1], of which kv_lens[s] are valid, all if kv_lens is None).  Returns (o[Tq,Hq,d], lse[Hq,Tq] fp32);
    a sequence without valid keys gets o = 0, lse = -inf.  Work goes to `stream`, by default the current one of q's device; so do the
    tensors that are made here."""
    Tq, Tk, nseq, hq, hkv, d, dt, ws = _cross_sizes(q, k, v, cu_q, cu_kv, max_seqlen_q, max_seqlen_kv, workspace, False, stream)
    dev = q.device
    o = _like("out", out, q.shape, q.dtype, dev, stream)
    lse = _like("lse", lse, (hq, Tq), torch.float32, dev, stream)
    kq, hp_q = _host_lens("cu_q_host", cu_q_host, nseq)
    kk, hp_k = _host_lens("cu_kv_host", cu_kv_host, nseq)
    _on_device(dev, load().hyd_cross_attn_fwd,
               (q.data_ptr(), k.data_ptr(), v.data_ptr(), _int32("cu_q", cu_q, nseq + 1, dev), _int32("cu_kv", cu_kv, nseq + 1, dev),
                _int32("kv_lens", kv_lens, nseq, dev), nseq, hp_q, hp_k, Tq, Tk, int(max_seqlen_q), int(max_seqlen_kv), hq, hkv, d,
                float(softmax_scale), dt, o.data_ptr(), lse.data_ptr(), ws.data_ptr(), ws.numel()), stream)
    return o, lse


def cross_attn_bwd(q, k, v, o, lse, d_o, cu_q, cu_kv, max_seqlen_q, max_seqlen_kv, softmax_scale, kv_lens=None, cu_q_host=None,
                   cu_kv_host=None, workspace=None, stream=None, dq=None, dk=None, dv=None):
    """Gradients (dq, dk, dv) of cross_attn_fwd for an upstream gradient d_o of o; o and lse are the forward's results.  Rows of dk
    and dv behind a sequence's valid keys are zeros."""
    Tq, Tk, nseq, hq, hkv, d, dt, ws = _cross_sizes(q, k, v, cu_q, cu_kv, max_seqlen_q, max_seqlen_kv, workspace, True, stream)
    dev = q.device
    _like("o", o, q.shape, q.dtype, dev)
    _like("d_o", d_o, q.shape, q.dtype, dev)
    _like("lse", lse, (hq, Tq), torch.float32, dev)
    dq = _like("dq", dq, q.shape, q.dtype, dev, stream)
    dk = _like("dk", dk, k.shape, k.dtype, dev, stream)
    dv = _like("dv", dv, v.shape, v.dtype, dev, stream)
    kq, hp_q = _host_lens("cu_q_host", cu_q_host, nseq)
    kk, hp_k = _host_lens("cu_kv_host", cu_kv_host, nseq)
    _on_device(dev, load().hyd_cross_attn_bwd,
               (q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr(), d_o.data_ptr(), _int32("cu_q", cu_q, nseq + 1, dev),
                _int32("cu_kv", cu_kv, nseq + 1, dev), _int32("kv_lens", kv_lens, nseq, dev), nseq, hp_q, hp_k, Tq, Tk, int(max_seqlen_q),
                int(max_seqlen_kv), hq, hkv, d, float(softmax_scale), dt, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(),
                ws.numel()), stream)
    return dq, dk, dv


def rope_frequencies(rot_dim, base=10000.0, scaling="plain", factor=1.0, original_length=0.0, low=1.0, high=32.0, device="cuda"):
    """Frequencies of the rot_dim / 2 pairs for rope_rotate, as a float64 tensor on `device`: made once per model.  `scaling`:
    "plain", "linear" or "parts" (see hyd_rope_frequencies)."""
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(ROPE_SCALINGS)}, got {scaling!r}")
    out = np.zeros(max(int(rot_dim) // 2, 1), dtype=np.float64)
    _check(load().hyd_rope_frequencies(int(rot_dim), float(base), ROPE_SCALINGS[scaling], float(factor), float(original_length),
                                       float(low), float(high), out.ctypes.data))
    return torch.from_numpy(out).to(device)


def _rope_tensor(name, x, out, T, d, dt, device, stream):
    """Checks a tensor of rope_rotate and its output (made if None), [T, heads, d] with the heads of a token contiguous: (output,
    heads, the tensor's token stride, the output's)."""
    shape = x.shape
    if len(shape) != 3 or shape[0] != T or shape[2] != d or x.dtype != dt or x.device != device:
        raise ValueError(f"{name} must be [{T}, heads, {d}] in {dt} on {device}, got {tuple(shape)} {x.dtype} {x.device}")
    if out is None:
        out = _made(shape, dt, device, stream)
    elif out.shape != shape or out.dtype != dt or out.device != device:
        raise ValueError(f"the output of {name} must be like it, got {tuple(out.shape)} {out.dtype} {out.device}")
    heads = shape[1]
    token = []
    for t in (x, out):
        st = t.stride()
        if T and ((d > 1 and st[2] != 1) or (heads > 1 and st[1] != d) or (T > 1 and st[0] < heads * d)):
            raise ValueError(f"{name}: the heads of a token must be contiguous, got strides {st}")
        token.append(st[0] if T > 1 else heads * d)
    return out, heads, token[0], token[1]


def _int32(name, t, n, device):
    """A device int32 tensor of n elements (or None) as a pointer."""
    if t is None:
        return None
    if t.dtype != torch.int32 or not t.is_contiguous() or t.numel() != n or t.device != device:
        raise ValueError(f"{name} must be a contiguous int32 tensor of {n} elements on {device}, got {t.dtype} {tuple(t.shape)} {t.device}")
    return t.data_ptr()


def rope_rotate(q, freqs, k=None, cu_seqlens=None, starts=None, positions=None, layout="half", magnitude=1.0, inverse=False,
                out=None, k_out=None, stream=None):
    """Rotary positions on q[T,H,d] and, with k[T,Hk,d], on both in one launch (bf16 or fp32, the rows may be strided); the first
    2 * freqs.numel() elements of every head are turned.  The rows' positions are `positions` (int32 [T]) or follow from
    cu_seqlens (int32 [num_seqs+1]) and `starts` (int32 [num_seqs] or None).  out may be q, k_out may be k.  Returns out, or
    (out, k_out).  Work goes to `stream`, by default the current one of q's device; so do the tensors that are made here."""
    if q.dim() != 3:
        raise ValueError(f"q must be [T, heads, d], got {tuple(q.shape)}")
    T, hq, d = q.shape
    dt, dev = _dtype_code(q), q.device
    if layout not in ROPE_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(ROPE_LAYOUTS)}, got {layout!r}")
    if freqs.dtype != torch.float64 or not freqs.is_contiguous() or freqs.device != dev:
        raise ValueError(f"freqs must be a contiguous float64 tensor on {dev}, got {freqs.dtype} {freqs.device}")
    if (cu_seqlens is None) == (positions is None):
        raise ValueError("either cu_seqlens or positions")
    if starts is not None and cu_seqlens is None:
        raise ValueError("starts go with cu_seqlens")
    nseq = 0 if cu_seqlens is None else cu_seqlens.numel() - 1
    if nseq < 0:
        raise ValueError("cu_seqlens must have num_seqs + 1 elements")
    out, hq, qs, qos = _rope_tensor("q", q, out, T, d, q.dtype, dev, stream)
    kp, kop, hk, ks, kos = None, None, 0, 0, 0
    if k is not None:
        k_out, hk, ks, kos = _rope_tensor("k", k, k_out, T, d, q.dtype, dev, stream)
        kp, kop = k.data_ptr(), k_out.data_ptr()
    _on_device(dev, load().hyd_rope_rotate,
               (q.data_ptr(), hq, qs, out.data_ptr(), qos, kp, hk, ks, kop, kos, _int32("cu_seqlens", cu_seqlens, nseq + 1, dev),
                _int32("starts", starts, nseq, dev), nseq, _int32("positions", positions, T, dev), T, d, freqs.data_ptr(),
                2 * freqs.numel(), ROPE_LAYOUTS[layout], float(magnitude), int(bool(inverse)), dt), stream)
    return out if k is None else (out, k_out)


def enable_kernel_timing(on):
    load().hyd_enable_kernel_timing(int(bool(on)))


def kernel_times(cap=8192):
    """[(kernel name, milliseconds)] in launch order of every kernel enqueued since timing was
    enabled or since the previous call of this function; synchronises on them and empties the list."""
    names = (ctypes.c_char_p * cap)()
    ms = (ctypes.c_float * cap)()
    n = load().hyd_kernel_times(names, ms, cap)
    return [(names[i].decode(), float(ms[i])) for i in range(n)]


def set_wg_trace(records):
    """records: int64 device tensor [3 * per_kernel, 4] (or None to switch the trace off)."""
    if records is None:
        load().hyd_set_wg_trace(None, 0)
    else:
        assert records.dtype == torch.int64 and records.is_contiguous() and records.shape[1] == 4
        load().hyd_set_wg_trace(records.data_ptr(), records.shape[0])


def schedule_status(workspace, total_tokens, num_seqs, hq, hkv, head_dim, dtype_code, is_bwd, stream=None):
    """Status code of what the last call's schedule prelude saw in the device cu_seqlens
    (synchronises the stream): 0, HYD_ERR_SHAPE (2) or HYD_ERR_SEQLENS (6)."""
    return int(load().hyd_varlen_attn_schedule_status(workspace.data_ptr(), workspace.numel(), total_tokens, num_seqs, hq, hkv,
                                                      head_dim, dtype_code, int(is_bwd), _stream_ptr(stream)))


def schedule_items(workspace, total_tokens, num_seqs, hq, hkv, head_dim, dtype_code, is_bwd, which):
    """The item list a finished call left in `workspace`: (tile, int array [n, 4] of (sequence,
    level, first packed row, length)), copied to the host."""
    hdr, items, cap, tile = ctypes.c_size_t(0), ctypes.c_size_t(0), ctypes.c_int(0), ctypes.c_int(0)
    _check(load().hyd_varlen_attn_schedule_layout(total_tokens, num_seqs, hq, hkv, head_dim, dtype_code, int(is_bwd), int(which),
                                                  ctypes.byref(hdr), ctypes.byref(items), ctypes.byref(cap), ctypes.byref(tile)))
    torch.cuda.synchronize()
    n = int(workspace[hdr.value:hdr.value + 4].view(torch.int32).item())
    assert 0 <= n <= cap.value
    rec = workspace[items.value:items.value + 16 * n].view(torch.int32).reshape(n, 4).cpu().numpy()
    return tile.value, rec


def executed_items(workspace, total_tokens, num_seqs, hq, hkv, head_dim, dtype_code, is_bwd, which):
    """The records that the kernel of a finished call took, in the order in which they were handed out: (rows of a
    tile, heads of a record, int array [n, 6] of (sequence, level, first packed row, length, part, parts))."""
    hdr, items, cap, tile = ctypes.c_size_t(0), ctypes.c_size_t(0), ctypes.c_int(0), ctypes.c_int(0)
    _check(load().hyd_varlen_attn_schedule_layout(total_tokens, num_seqs, hq, hkv, head_dim, dtype_code, int(is_bwd), int(which),
                                                  ctypes.byref(hdr), ctypes.byref(items), ctypes.byref(cap), ctypes.byref(tile)))
    torch.cuda.synchronize()
    words = lambda at, n: workspace[at:at + 4 * n].view(torch.int32).cpu().numpy()
    at = hdr.value + int(words(hdr.value, 4)[3])
    h = words(at, 7)
    rec = words(at + int(h[4]), 4 * int(h[2])).reshape(-1, 4)
    level, part, parts = rec[:, 1] & 0xffffff, (rec[:, 1] >> 24) & 7, ((rec[:, 1] >> 27) & 7) + 1
    return int(h[5]), int(h[6]), np.column_stack([rec[:, 0], level, rec[:, 2], rec[:, 3], part, parts])
