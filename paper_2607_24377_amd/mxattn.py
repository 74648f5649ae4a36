"""ctypes binding of libmxattn (include/mxattn.h).

Argument marshalling only: every step of the hot path runs in the HIP
library.  PyTorch provides device memory and the current stream.  There is no
CPU fallback; if ``libmxattn.so`` is missing or cannot be loaded, every call
raises.
"""
from __future__ import annotations

import ctypes
import os
import threading
from array import array

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmxattn.so")

MODES = {"ocp_vanilla": 0, "uos": 1, "uos_pnq": 2, "uos_pnq_rot": 3}
AXIS_TOKENS, AXIS_HEAD_DIM = 2, 3
OK = 0
WITH_DETAIL = (7, 8, 10)  # out of memory, a HIP error, too little scratch

_lock = threading.Lock()
_lib = None


class MxattnError(RuntimeError):
    def __init__(self, status: int, where: str):
        L = lib()
        msg = L.mxattn_status_string(status).decode()
        # (the detail is of the last error that had one: of another call, where this status has none)
        detail = L.mxattn_last_error().decode() if status in WITH_DETAIL else ""
        super().__init__(f"{where}: status {status} ({msg}){': ' + detail if detail else ''}")
        self.status = status


def lib() -> ctypes.CDLL:
    """Load libmxattn.so (built in-tree by ``python -m paper_2607_24377_amd.build``)."""
    global _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise RuntimeError(
                    f"{LIB_PATH} is missing: build it with `python -m paper_2607_24377_amd.build`")
            L = ctypes.CDLL(LIB_PATH)
            P, I, I64, SZ = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
            L.mxattn_quantize.argtypes = [P, P, P, I, I, I64, I64, I64, I64, P]
            L.mxattn_quantize.restype = I
            D = ctypes.c_double
            L.mxattn_quantize_qmax.argtypes = [P, P, P, I, D, I64, I64, I64, I64, P]
            L.mxattn_quantize_qmax.restype = I
            L.mxattn_qmax_sse.argtypes = [P, I, P, I, P, I64, I64, I64, I64, P]
            L.mxattn_qmax_sse.restype = I
            F = ctypes.c_float
            L.mxattn_softmax_rows.argtypes = [P, P, P, I64, I64, I64, I64, I64, I64, I64, I64, P]
            L.mxattn_softmax_rows.restype = I
            L.mxattn_rowsum_diag.argtypes = [P, I64, I64, I64, I, F, P, P]
            L.mxattn_rowsum_diag.restype = I
            L.mxattn_attention_rowsum_diag.argtypes = [P, P, I64, I64, I64, I64, I64, I, F, P, P]
            L.mxattn_attention_rowsum_diag.restype = I
            L.mxattn_forward.argtypes = [P, P, P, P, I64, I64, I64, I64, I, P]
            L.mxattn_forward.restype = I
            L.mxattn_attend.argtypes = [P, P, P, P, P, P, P, I64, I64, I64, I64, I, P]
            L.mxattn_cross_forward.argtypes = [P, P, P, P, I64, I64, I64, I64, I64, I, P]
            L.mxattn_cross_forward.restype = I
            L.mxattn_cross_attend.argtypes = [P, P, P, P, P, P, P, I64, I64, I64, I64, I64, I, P]
            L.mxattn_cross_attend.restype = I
            L.mxattn_cross_attend_noalloc.argtypes = [P, P, P, P, P, P, P, I64, I64, I64, I64, I64, I, P]
            L.mxattn_cross_attend_noalloc.restype = I
            L.mxattn_attend.restype = I
            L.mxattn_qk_norm_rope.argtypes = [P, P, P, P, I64, I64, I64, I64, I64, P, P, P, P, P, P, F, P, P, P,
                                              I64, I64, I, P]
            L.mxattn_qk_norm_rope.restype = I
            L.mxattn_cache_append.argtypes = [P, P, I64, I64, P, P, P, P, I64, I64, P, P, P, I64, I64, I64, I64, I64,
                                              P, F, P, P, P, I64, I64, I, P]
            L.mxattn_cache_append.restype = I
            L.mxattn_cache_attend.argtypes = [P, I64, P, P, P, P, I64, I64, P, P, P, I64, I64, I64, I64, I64, I64, I,
                                              I64, I64, P, I64, P, SZ, P]
            L.mxattn_cache_attend.restype = I
            L.mxattn_cache_attend_workspace.argtypes = [I64] * 8
            L.mxattn_cache_attend_workspace.restype = SZ
            batch = [P, I64, P, P, P, P, I64, I64, P, P, P, I64, I64, I64, I64, I64, I64]
            L.mxattn_cache_attend_window.argtypes = batch + [I64, I64, I, I64, I64, P, I64, P, SZ, P]
            L.mxattn_cache_attend_window.restype = I
            L.mxattn_cache_attend_tree.argtypes = batch + [P, I64, I64, I64, P, I64, P, SZ, P]
            L.mxattn_cache_attend_tree.restype = I
            L.mxattn_cache_attend_weights.argtypes = batch + [P, P, I, I64, I64, P, I64, P, SZ, P]
            L.mxattn_cache_attend_weights.restype = I
            L.mxattn_cache_attend_weights_workspace.argtypes = [I64] * 8
            L.mxattn_cache_attend_weights_workspace.restype = SZ
            L.mxattn_cache_select.argtypes = [P, I64, I64, P, P] + [I64] * 6 + [P, P, P, SZ, P]
            L.mxattn_cache_select_workspace.argtypes = [I64] * 4
            L.mxattn_cache_select_workspace.restype = SZ
            L.mxattn_cache_select.restype = I
            L.mxattn_cache_compact.argtypes = [P, P, P, P, I64, I64, P, I64, I64, P, I64, I64, I64, P, I64, I64, P, P, P, P]
            L.mxattn_cache_compact.restype = I
            L.mxattn_codes_bytes.argtypes = [I, I64, I64, I64, I64]
            L.mxattn_codes_bytes.restype = SZ
            L.mxattn_scales_bytes.argtypes = [I, I64, I64, I64, I64]
            L.mxattn_scales_bytes.restype = SZ
            L.mxattn_kv_tile.argtypes = []
            L.mxattn_kv_tile.restype = I
            L.mxattn_query_tile.argtypes = []
            L.mxattn_query_tile.restype = I
            L.mxattn_status_string.argtypes = [I]
            L.mxattn_status_string.restype = ctypes.c_char_p
            L.mxattn_last_error.argtypes = []
            L.mxattn_last_error.restype = ctypes.c_char_p
            L.mxattn_release_workspace.argtypes = []
            L.mxattn_release_workspace.restype = I
            L.mxattn_version.argtypes = []
            L.mxattn_version.restype = I
            _lib = L
    return _lib


def _mode(mode) -> int:
    return MODES[mode] if isinstance(mode, str) else int(mode)


def _stream(stream) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _empty(shape, dtype, device, stream):
    """Memory for what a call writes.  On a stream that is given it is that stream's: what the current stream's
    allocator has free may still be in use by work enqueued there.  It is not reused before the current stream, where
    the caller has the tensor, is done with it either."""
    if stream is not None:
        here, there = torch.cuda.current_stream(device), _stream(stream)
        if there != here.cuda_stream:
            with torch.cuda.stream(torch.cuda.ExternalStream(there, device)):
                t = torch.empty(shape, dtype=dtype, device=device)
            t.record_stream(here)
            return t
    return torch.empty(shape, dtype=dtype, device=device)


def _check(st: int, where: str):
    if st != OK:
        raise MxattnError(st, where)


def kv_tile() -> int:
    return lib().mxattn_kv_tile()


def query_tile() -> int:
    return lib().mxattn_query_tile()


def code_shapes(block_axis: int, B: int, H: int, N: int, d: int = 128):
    """Shapes of the codes and scales arrays of a [B, H, N, d] tensor."""
    if block_axis == AXIS_HEAD_DIM:
        return (B, H, N, d // 2), (B, H, N, d // 32)
    nb = (N + 31) // 32
    return (B, H, d, nb * 16), (B, H, d, nb)


def _bhnd(x: torch.Tensor):
    if x.dim() != 4:
        raise ValueError("expected a [B, H, N, d] tensor")
    if x.dtype != torch.bfloat16 or not x.is_cuda or not x.is_contiguous():
        raise ValueError("expected a contiguous bf16 CUDA tensor")
    return x.shape


def quantize(x: torch.Tensor, block_axis: int, mode, stream=None, codes=None, scales=None):
    """MXFP4-quantize bf16 x [B, H, N, d]; returns (codes, scales) uint8 tensors."""
    B, H, N, d = _bhnd(x)
    cs, ss = code_shapes(block_axis, B, H, N, d)
    if codes is None:
        codes = _empty(cs, torch.uint8, x.device, stream)
    if scales is None:
        scales = _empty(ss, torch.uint8, x.device, stream)
    st = lib().mxattn_quantize(x.data_ptr(), codes.data_ptr(), scales.data_ptr(), block_axis,
                               _mode(mode), B, H, N, d, _stream(stream))
    _check(st, "mxattn_quantize")
    return codes, scales


def quantize_qmax(x: torch.Tensor, block_axis: int, qmax: float, stream=None, codes=None, scales=None):
    """MXFP4-quantize bf16 x [B, H, N, d] with the ceil rule of boundary qmax."""
    B, H, N, d = _bhnd(x)
    cs, ss = code_shapes(block_axis, B, H, N, d)
    if codes is None:
        codes = _empty(cs, torch.uint8, x.device, stream)
    if scales is None:
        scales = _empty(ss, torch.uint8, x.device, stream)
    st = lib().mxattn_quantize_qmax(x.data_ptr(), codes.data_ptr(), scales.data_ptr(), block_axis,
                                    float(qmax), B, H, N, d, _stream(stream))
    _check(st, "mxattn_quantize_qmax")
    return codes, scales


def qmax_sse(x: torch.Tensor, block_axis: int, qs, stream=None, out=None):
    """Per-(batch, head) sum of squared MXFP4 errors of bf16 x [B, H, N, d] for
    each boundary in qs; returns a float64 device tensor [B*H, len(qs)]."""
    B, H, N, d = _bhnd(x)
    q = (ctypes.c_double * len(qs))(*[float(v) for v in qs])
    if out is None:
        out = _empty((B * H, len(qs)), torch.float64, x.device, stream)
    st = lib().mxattn_qmax_sse(x.data_ptr(), block_axis, ctypes.cast(q, ctypes.c_void_p), len(qs),
                               out.data_ptr(), B, H, N, d, _stream(stream))
    _check(st, "mxattn_qmax_sse")
    return out


DIAG_FIELDS = ("rowsum", "mass", "zeroing", "saturation", "down", "up", "exact", "entropy")


def softmax_rows(q: torch.Tensor, k: torch.Tensor, row0: int = 0, rows: int | None = None, ld=None,
                 stream=None, out=None):
    """fp32 softmax(q k^T / sqrt(d)) for query rows [row0, row0 + rows) of
    every head: [B, H, rows, ld] (ld = Nkv rounded up to 4; entries past Nkv
    are left as allocated)."""
    B, H, Nq, d = _bhnd(q)
    Bk, Hk, Nkv, dk = _bhnd(k)
    if (Bk, Hk, dk) != (B, H, d):
        raise ValueError("k must be [B, H, Nkv, d] with q's B, H, d")
    rows = Nq - row0 if rows is None else rows
    ld = (Nkv + 3) // 4 * 4 if ld is None else ld
    if out is None:
        out = _empty((B, H, rows, ld), torch.float32, q.device, stream)
    st = lib().mxattn_softmax_rows(q.data_ptr(), k.data_ptr(), out.data_ptr(), B, H, Nq, Nkv, d, row0,
                                   rows, ld, _stream(stream))
    _check(st, "mxattn_softmax_rows")
    return out


def rowsum_diag(p: torch.Tensor, N: int, mode, gamma: float = 1.0, stream=None, out=None):
    """Row-sum diagnostics of fp32 rows p [..., ld] (first N entries): [rows, 8]
    float64 in DIAG_FIELDS order."""
    if p.dtype != torch.float32 or not p.is_cuda or not p.is_contiguous():
        raise ValueError("expected a contiguous fp32 CUDA tensor")
    ld = p.shape[-1]
    rows = p.numel() // ld
    if out is None:
        out = _empty((rows, 8), torch.float64, p.device, stream)
    st = lib().mxattn_rowsum_diag(p.data_ptr(), rows, N, ld, _mode(mode), float(gamma), out.data_ptr(),
                                  _stream(stream))
    _check(st, "mxattn_rowsum_diag")
    return out


def attention_rowsum_diag(q: torch.Tensor, k: torch.Tensor, mode, gamma: float = 1.0, stream=None,
                          out=None):
    """Row-sum diagnostics of every attention row: [B, H, Nq, 8] float64."""
    B, H, Nq, d = _bhnd(q)
    Bk, Hk, Nkv, dk = _bhnd(k)
    if (Bk, Hk, dk) != (B, H, d):
        raise ValueError("k must be [B, H, Nkv, d] with q's B, H, d")
    if out is None:
        out = _empty((B, H, Nq, 8), torch.float64, q.device, stream)
    st = lib().mxattn_attention_rowsum_diag(q.data_ptr(), k.data_ptr(), B, H, Nq, Nkv, d, _mode(mode),
                                            float(gamma), out.data_ptr(), _stream(stream))
    _check(st, "mxattn_attention_rowsum_diag")
    return out


def forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, mode, out=None, stream=None):
    """MXFP4 attention forward of bf16 q, k, v [B, H, N, d]; returns bf16 out."""
    B, H, N, d = _bhnd(q)
    if _bhnd(k) != q.shape or _bhnd(v) != q.shape:
        raise ValueError("q, k, v must have the same shape")
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    st = lib().mxattn_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H, N, d,
                              _mode(mode), _stream(stream))
    _check(st, "mxattn_forward")
    return out


def attend(qc, qs, kc, ks, vc, vs, N: int, mode, out=None, stream=None):
    """The fused kernel on quantized operands (library layouts); returns bf16 out."""
    B, H = qc.shape[0], qc.shape[1]
    d = qc.shape[3] * 2
    if out is None:
        out = _empty((B, H, N, d), torch.bfloat16, qc.device, stream)
    st = lib().mxattn_attend(qc.data_ptr(), qs.data_ptr(), kc.data_ptr(), ks.data_ptr(),
                             vc.data_ptr(), vs.data_ptr(), out.data_ptr(), B, H, N, d, _mode(mode),
                             _stream(stream))
    _check(st, "mxattn_attend")
    return out


def cross_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, mode, out=None, stream=None):
    """Attention of bf16 q [B, H, Nq, d] over k, v [B, H, Nkv, d]; returns bf16 out [B, H, Nq, d]."""
    B, H, Nq, d = _bhnd(q)
    Bk, Hk, Nkv, dk = _bhnd(k)
    if (Bk, Hk, dk) != (B, H, d) or _bhnd(v) != k.shape:
        raise ValueError("k and v must be [B, H, Nkv, d] with q's B, H, d")
    if out is None:
        out = _empty(q.shape, q.dtype, q.device, stream)
    st = lib().mxattn_cross_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H,
                                    Nq, Nkv, d, _mode(mode), _stream(stream))
    _check(st, "mxattn_cross_forward")
    return out


def cross_attend(qc, qs, kc, ks, vc, vs, Nq: int, Nkv: int, mode, out=None, stream=None):
    """The fused kernel on quantized operands with Nq queries and Nkv keys."""
    B, H = qc.shape[0], qc.shape[1]
    d = qc.shape[3] * 2
    if out is None:
        out = _empty((B, H, Nq, d), torch.bfloat16, qc.device, stream)
    st = lib().mxattn_cross_attend(qc.data_ptr(), qs.data_ptr(), kc.data_ptr(), ks.data_ptr(),
                                   vc.data_ptr(), vs.data_ptr(), out.data_ptr(), B, H, Nq, Nkv, d,
                                   _mode(mode), _stream(stream))
    _check(st, "mxattn_cross_attend")
    return out


PAIRS = {"interleaved": 0, "halves": 1}
BLOCK_TOKENS = 32


def _raw_stream(index: int) -> int:
    """The device's current stream.  The public call takes 4 us to make an object of it; a torch without the other has
    that one."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw else torch.cuda.current_stream(index).cuda_stream


def _run(fn, where: str, index: int, stream, args):
    """fn(*args, stream) with device `index` current, on its current stream unless one is given."""
    if index == torch.cuda.current_device():
        st = fn(*args, _raw_stream(index) if stream is None else _stream(stream))
    else:
        with torch.cuda.device(index):
            st = fn(*args, _raw_stream(index) if stream is None else _stream(stream))
    if st != OK:
        raise MxattnError(st, where)


def _address(t, name, dtype, index, numel):
    """The address of t, contiguous and of so many elements on device `index`; NULL for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != numel or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} CUDA tensor of {numel} elements on device {index}")
    return t.data_ptr()


def _index(t, name) -> int:
    if t.dtype is not torch.bfloat16 or not t.is_cuda:
        raise ValueError(f"{name} must be a bf16 CUDA tensor")
    return t.get_device()


def _heads(t, name, index):
    """Address and strides (an array; None: contiguous) of a bf16 [B, H, N, d] tensor with contiguous channels."""
    if t.dim() != 4 or t.dtype is not torch.bfloat16 or t.get_device() != index:
        raise ValueError(f"{name} must be a bf16 [B, H, N, d] CUDA tensor on device {index}")
    if t.is_contiguous():
        return t.data_ptr(), None
    strides = array("q", t.stride())
    if strides[3] != 1:
        raise ValueError(f"{name}'s channels must be contiguous")
    return t.data_ptr(), strides


def _items(strides):
    return None if strides is None else strides.buffer_info()[0]


def _tables(cos, sin, index):
    """Addresses, rows and rotated channels of cos, sin [rows, rot / 2]; no rotation without them."""
    if cos is None and sin is None:
        return None, None, 0, 0
    if cos is None or sin is None or cos.dim() != 2 or sin.dim() != 2:
        raise ValueError("cos and sin must both be given, [rows, rot / 2]")
    rows, half = cos.shape
    if sin.size(1) != half:
        raise ValueError("sin must have cos's shape")
    f32 = torch.float32
    return (_address(cos, "cos", f32, index, rows * half), _address(sin, "sin", f32, index, rows * half), rows, 2 * half)


def _pairs(pairs) -> int:
    return PAIRS[pairs] if isinstance(pairs, str) else int(pairs)


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor | None, q_weight=None, k_weight=None, eps: float = 1e-6, cos=None,
                 sin=None, positions=None, pairs="interleaved", q_out=None, k_out=None, stream=None):
    """RMS norm of every head of bf16 q [B, Hq, N, d] and k [B, Hkv, N, d] (any strides; fp32 weights [d], None: no
    norm) and their rotation by position (fp32 cos, sin [rows, rot / 2]; int32 positions [B, N], None: 0 .. N - 1);
    returns (q_out, k_out), contiguous unless given.  k None: q alone."""
    dev = _index(q, "q")
    qp, qs = _heads(q, "q", dev)
    B, Hq, N, d = q.shape
    if q_out is None:
        q_out = _empty((B, Hq, N, d), q.dtype, q.device, stream)
        qop, qos = q_out.data_ptr(), None
    elif q_out.shape != q.shape:
        raise ValueError("q_out must have q's shape")
    else:
        qop, qos = _heads(q_out, "q_out", dev)
    kp = ks = kop = kos = None
    Hkv = 0
    if k is not None:
        kp, ks = _heads(k, "k", dev)
        Hkv = k.shape[1]
        if k.shape != (B, Hkv, N, d):
            raise ValueError("k must be [B, Hkv, N, d] with q's B, N, d")
        if k_out is None:
            k_out = _empty((B, Hkv, N, d), q.dtype, q.device, stream)
            kop = k_out.data_ptr()
        elif k_out.shape != k.shape:
            raise ValueError("k_out must have k's shape")
        else:
            kop, kos = _heads(k_out, "k_out", dev)
    elif k_out is not None or k_weight is not None:
        raise ValueError("k_out and k_weight go with k")
    cp, sp, rows, rot = _tables(cos, sin, dev)
    f32 = torch.float32
    _run((_lib or lib()).mxattn_qk_norm_rope, "mxattn_qk_norm_rope", dev, stream,
         (qp, kp, qop, kop, B, Hq, Hkv, N, d, _items(qs), _items(ks), _items(qos), _items(kos),
          _address(q_weight, "q_weight", f32, dev, d),
          _address(k_weight, "k_weight", f32, dev, d), eps, cp, sp,
          _address(positions, "positions", torch.int32, dev, B * N), rows, rot, _pairs(pairs)))
    return q_out, k_out


def cache_shapes(pages: int, heads: int, page_tokens: int, d: int = 128):
    """Shapes of the uint8 arrays of a paged cache: K codes, K scales, V codes, V scales."""
    if d != 128 or not 32 <= page_tokens <= 4096 or page_tokens & (page_tokens - 1):
        raise ValueError("a cache has d = 128 and pages of a power of two from 32 to 4096 tokens")
    n = page_tokens // BLOCK_TOKENS
    scales = (pages, heads, n)
    return scales + (d // 16, BLOCK_TOKENS, 16), scales, scales + (d, BLOCK_TOKENS), scales


def _token_rows(t, name, index):
    """Address and token stride of a bf16 [tokens, heads, d] tensor with contiguous heads."""
    if t.dim() != 3 or t.dtype is not torch.bfloat16 or t.get_device() != index:
        raise ValueError(f"{name} must be a bf16 [tokens, heads, d] CUDA tensor on device {index}")
    stride, head, channel = t.stride()
    if channel != 1 or (head != t.shape[2] and t.shape[1] != 1):
        raise ValueError(f"{name}'s heads and channels must be contiguous")
    return t.data_ptr(), stride


def _cache_arrays(k_codes, v_codes, d):
    """Pages, heads and blocks per page of a cache's code arrays, which must agree."""
    pages, heads, blocks, *block = k_codes.shape
    if block != [d // 16, BLOCK_TOKENS, 16] or v_codes.shape != (pages, heads, blocks, d, BLOCK_TOKENS):
        raise ValueError(f"k_codes and v_codes must have the shapes of cache_shapes for heads of {d} channels")
    return pages, heads, blocks


def _cache(k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len, index, d):
    """Checked addresses and sizes of a cache of d channels and its batch, as the library takes them, and the cache's
    heads."""
    if k_codes.dim() != 6 or page_table.dim() != 2:
        raise ValueError("k_codes must be [pages, heads, page_tokens / 32, 8, 32, 16], page_table [seqs, max_pages]")
    pages, heads, blocks = _cache_arrays(k_codes, v_codes, d)
    seqs, max_pages = page_table.shape
    u8, i32, n = torch.uint8, torch.int32, pages * heads * blocks
    codes = n * d * BLOCK_TOKENS
    return (_address(k_codes, "k_codes", u8, index, codes), _address(k_scales, "k_scales", u8, index, n),
            _address(v_codes, "v_codes", u8, index, codes), _address(v_scales, "v_scales", u8, index, n), pages,
            blocks * BLOCK_TOKENS, _address(page_table, "page_table", i32, index, seqs * max_pages),
            _address(q_start, "q_start", i32, index, seqs + 1), _address(kv_len, "kv_len", i32, index, seqs), seqs,
            max_pages), heads


def cache_append(k: torch.Tensor, v: torch.Tensor, k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len,
                 k_weight=None, eps: float = 1e-6, cos=None, sin=None, positions=None, pairs="interleaved", stream=None):
    """Append bf16 k, v [tokens, Hkv, d] to a paged cache (arrays of cache_shapes): k normed and rotated as by
    qk_norm_rope on the way (int32 positions [tokens], None: a token's place in its sequence).  The call's tokens
    q_start[s] .. q_start[s + 1] - 1 are the last ones of the kv_len[s] of sequence s."""
    dev = _index(k, "k")
    (kp, kst), (vp, vst) = _token_rows(k, "k", dev), _token_rows(v, "v", dev)
    tokens, _, d = k.shape
    cache, heads = _cache(k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len, dev, d)
    if v.shape != k.shape or k.shape[1] != heads:
        raise ValueError("k and v must be [tokens, Hkv, d] with the cache's heads")
    cp, sp, rows, rot = _tables(cos, sin, dev)
    _run((_lib or lib()).mxattn_cache_append, "mxattn_cache_append", dev, stream,
         (kp, vp, kst, vst, *cache, tokens, heads, d, _address(k_weight, "k_weight", torch.float32, dev, d), eps, cp, sp,
          _address(positions, "positions", torch.int32, dev, tokens), rows, rot, _pairs(pairs)))


def cache_attend(q: torch.Tensor, k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len, causal: bool = True,
                 max_q: int = 0, max_kv: int = 0, out=None, stream=None):
    """Attention of bf16 q [tokens, Hq, d] over the sequences' cached keys; returns bf16 out [tokens, Hq, d].
    max_q, max_kv: at least the new tokens and the keys of every sequence as the caller knows them (0: unknown); they
    choose how the work is divided.  Wrong ones cost time, and other ones (or other lengths in the batch) may change an
    output by the rounding of the probabilities to f16.  Workspace is torch's, of the current stream (a graph
    captured there keeps it); of a stream that is given it is the library's, and a call that needs some cannot be
    captured."""
    return _attend("mxattn_cache_attend", q, (k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len), (causal,),
                   max_q, max_kv, out, stream)


def _attend(name, q, batch, middle, max_q, max_kv, out, stream, workspace="mxattn_cache_attend_workspace"):
    """Attention of q over a cache by the library's call `name`.  `middle`: its arguments between the batch's sizes and
    the bounds, or a function that checks them and gives them."""
    dev = _index(q, "q")
    qp, qst = _token_rows(q, "q", dev)
    tokens, Hq, d = q.shape
    cache, heads = _cache(*batch, dev, d)
    if callable(middle):
        middle = middle(dev, cache, heads, tokens)
    if out is None:
        out = _empty((tokens, Hq, d), q.dtype, q.device, stream)
    elif out.shape != q.shape:
        raise ValueError("out must have q's shape")
    op, ost = _token_rows(out, "out", dev)
    L, work, size = _lib or lib(), None, 0
    if stream is None:  # torch's memory belongs to the current stream, and to the graph that is captured on it
        size = getattr(L, workspace)(cache[5], *cache[9:], tokens, Hq, heads, max_q, max_kv)
        if size:
            work = torch.empty(size, dtype=torch.uint8, device=q.device)
    _run(getattr(L, name), name, dev, stream, (qp, qst, *cache, tokens, Hq, heads, d, *middle, max_q, max_kv, op, ost,
                                               work.data_ptr() if size else None, size))
    return out


def cache_attend_window(q: torch.Tensor, k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len, window: int,
                        sinks: int = 0, causal: bool = True, max_q: int = 0, max_kv: int = 0, out=None, stream=None):
    """cache_attend of the last `window` keys (of a token that sees T keys, positions T - window .. T - 1) and the
    first `sinks`.  Pages between that no token sees may have been given away: they are not read."""
    return _attend("mxattn_cache_attend_window", q, (k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len),
                   (window, sinks, causal), max_q, max_kv, out, stream)


def cache_attend_tree(q: torch.Tensor, k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len, tree,
                      max_q: int = 0, max_kv: int = 0, out=None, stream=None):
    """cache_attend for drafted tokens that form trees: a sequence's new token sees what was there before and those of
    its new tokens whose bit is set in its row of `tree`, int32 [tokens, words], bit j & 31 of word j >> 5 for new
    token j (its ancestors, and itself)."""
    def middle(dev, cache, heads, tokens):
        if tree.dim() != 2 or tree.shape[0] != tokens:
            raise ValueError("tree must be [tokens, words]")
        return _address(tree, "tree", torch.int32, dev, tree.numel()), tree.shape[1]

    return _attend("mxattn_cache_attend_tree", q, (k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len), middle,
                   max_q, max_kv, out, stream)


def _weights_shape(t, name, shape):
    if t.shape != shape:
        raise ValueError(f"{name} must be [pages, heads, page_tokens]: {list(shape)}")
    return t


def cache_attend_weights(q: torch.Tensor, k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len, weights=None,
                         causal: bool = True, max_q: int = 0, max_kv: int = 0, out=None, weights_out=None, stream=None):
    """cache_attend that also adds to every key's weight the probabilities that the new tokens and the heads of its
    group give it; new keys start at 0.  weights: fp32 [pages, Hkv, page_tokens] (None: zeros); weights_out: where
    the sums go (None: into `weights`, or a new tensor of zeros).  Returns (out, weights_out).  max_kv is a limit
    here: longer sequences count as impossible."""
    def middle(dev, cache, heads, tokens):
        nonlocal weights_out
        shape = (cache[4], heads, cache[5])
        if weights is not None:
            _weights_shape(weights, "weights", shape)
        if weights_out is None:
            if weights is None and stream is not None:  # (torch would clear it on another stream)
                raise ValueError("weights or weights_out must be given with a stream")
            weights_out = weights if weights is not None else torch.zeros(shape, dtype=torch.float32, device=q.device)
        n = cache[4] * heads * cache[5]
        return (_address(weights, "weights", torch.float32, dev, n),
                _address(_weights_shape(weights_out, "weights_out", shape), "weights_out", torch.float32, dev, n), causal)

    out = _attend("mxattn_cache_attend_weights", q, (k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len),
                  middle, max_q, max_kv, out, stream, "mxattn_cache_attend_weights_workspace")
    return out, weights_out


def cache_select(weights: torch.Tensor, page_table, kv_len, budget: int, sinks: int = 0, recent: int = 0, kept=None,
                 counts=None, stream=None):
    """Which tokens stay when every sequence is cut to `budget`, for each KV head of fp32 weights [pages, Hkv,
    page_tokens]: the first `sinks`, the last `recent` and the heaviest between (ties: the first).  Returns (kept
    int32 [seqs, Hkv, budget], ascending positions and -1 behind them; counts int32 [seqs])."""
    if weights.dim() != 3 or page_table.dim() != 2 or not weights.is_cuda:
        raise ValueError("weights must be a CUDA tensor [pages, heads, page_tokens], page_table [seqs, max_pages]")
    dev = weights.get_device()
    pages, heads, page = weights.shape
    seqs, max_pages = page_table.shape
    i32 = torch.int32
    if kept is None:
        kept = _empty((seqs, heads, max(budget, 0)), i32, weights.device, stream)
    elif kept.shape != (seqs, heads, budget):
        raise ValueError("kept must be [seqs, heads, budget]")
    if counts is None:
        counts = _empty((seqs,), i32, weights.device, stream)
    L, work, size = _lib or lib(), None, 0
    if stream is None:  # (as for attention)
        size = L.mxattn_cache_select_workspace(page, seqs, max_pages, heads)
        if size:
            work = torch.empty(size, dtype=torch.uint8, device=weights.device)
    _run(L.mxattn_cache_select, "mxattn_cache_select", dev, stream,
         (_address(weights, "weights", torch.float32, dev, weights.numel()), pages, page,
          _address(page_table, "page_table", i32, dev, seqs * max_pages), _address(kv_len, "kv_len", i32, dev, seqs), seqs,
          max_pages, heads, budget, sinks, recent, _address(kept, "kept", i32, dev, kept.numel()),
          _address(counts, "counts", i32, dev, seqs), work.data_ptr() if size else None, size))
    return kept, counts


def cache_compact(k_codes: torch.Tensor, k_scales, v_codes, v_scales, page_table, kept, counts, base=None, out_table=None,
                  weights=None, stream=None):
    """Move kept tokens together: position base + i (i < counts) of a sequence becomes what was at kept[.., i], in K, V
    and, if given, fp32 weights [pages, Hkv, page_tokens].  kept: int32 [seqs, Hkv or 1, width]; counts, base (None: 0):
    int32 [seqs].  out_table: the page table of where they go, pages that hold none of the sources; None: in place
    (kept ascending, kept[i] >= base + i; a head's blocks one after another, so for a few blocks).  Keys keep their
    rotation: tokens appended afterwards need `positions`, as their place in the sequence is no longer their position."""
    if not k_codes.is_cuda or k_codes.dim() != 6 or kept.dim() != 3:
        raise ValueError("k_codes must be a CUDA tensor as of cache_shapes, kept [seqs, heads or 1, width]")
    dev, d = k_codes.get_device(), 128
    seqs, kept_heads, width = kept.shape
    i32 = torch.int32
    # (the batch's starts and lengths are of no concern here: a table and counts are)
    pages, heads, blocks = _cache_arrays(k_codes, v_codes, d)
    if page_table.dim() != 2 or page_table.shape[0] != seqs:
        raise ValueError("page_table must be [seqs, max_pages], kept [seqs, heads or 1, width]")
    n = pages * heads * blocks
    u8, codes = torch.uint8, n * d * BLOCK_TOKENS
    if out_table is not None and (out_table.dim() != 2 or out_table.shape[0] != seqs):
        raise ValueError("out_table must be [seqs, pages]")
    if weights is not None:
        _weights_shape(weights, "weights", (pages, heads, blocks * BLOCK_TOKENS))
    _run((_lib or lib()).mxattn_cache_compact, "mxattn_cache_compact", dev, stream,
         (_address(k_codes, "k_codes", u8, dev, codes), _address(k_scales, "k_scales", u8, dev, n),
          _address(v_codes, "v_codes", u8, dev, codes), _address(v_scales, "v_scales", u8, dev, n), pages,
          blocks * BLOCK_TOKENS, _address(page_table, "page_table", i32, dev, page_table.numel()), seqs, page_table.shape[1],
          None if out_table is None else _address(out_table, "out_table", i32, dev, out_table.numel()),
          0 if out_table is None else out_table.shape[1], heads, d, _address(kept, "kept", i32, dev, kept.numel()),
          kept_heads, width, _address(counts, "counts", i32, dev, seqs), _address(base, "base", i32, dev, seqs),
          _address(weights, "weights", torch.float32, dev, n * BLOCK_TOKENS)))


def bf16_from_bits(bits, device="cuda") -> torch.Tensor:
    """bf16 tensor from a numpy uint16 array of bit patterns."""
    import numpy as np

    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.view(torch.bfloat16).to(device)


def bits_from_bf16(t: torch.Tensor):
    """numpy uint16 bit patterns of a bf16 tensor."""
    return t.detach().contiguous().cpu().view(torch.int16).numpy().view("uint16")


def release_workspace():
    """Return the current device's cached workspace (mxattn_release_workspace)."""
    _check(lib().mxattn_release_workspace(), "mxattn_release_workspace")
