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
        codes = torch.empty(cs, dtype=torch.uint8, device=x.device)
    if scales is None:
        scales = torch.empty(ss, dtype=torch.uint8, device=x.device)
    st = lib().mxattn_quantize(x.data_ptr(), codes.data_ptr(), scales.data_ptr(), block_axis,
                               _mode(mode), B, H, N, d, _stream(stream))
    _check(st, "mxattn_quantize")
    return codes, scales


def quantize_qmax(x: torch.Tensor, block_axis: int, qmax: float, stream=None, codes=None, scales=None):
    """MXFP4-quantize bf16 x [B, H, N, d] with the ceil rule of boundary qmax."""
    B, H, N, d = _bhnd(x)
    cs, ss = code_shapes(block_axis, B, H, N, d)
    if codes is None:
        codes = torch.empty(cs, dtype=torch.uint8, device=x.device)
    if scales is None:
        scales = torch.empty(ss, dtype=torch.uint8, device=x.device)
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
        out = torch.empty((B * H, len(qs)), dtype=torch.float64, device=x.device)
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
        out = torch.empty((B, H, rows, ld), dtype=torch.float32, device=q.device)
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
        out = torch.empty((rows, 8), dtype=torch.float64, device=p.device)
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
        out = torch.empty((B, H, Nq, 8), dtype=torch.float64, device=q.device)
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
        out = torch.empty_like(q)
    st = lib().mxattn_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H, N, d,
                              _mode(mode), _stream(stream))
    _check(st, "mxattn_forward")
    return out


def attend(qc, qs, kc, ks, vc, vs, N: int, mode, out=None, stream=None):
    """The fused kernel on quantized operands (library layouts); returns bf16 out."""
    B, H = qc.shape[0], qc.shape[1]
    d = qc.shape[3] * 2
    if out is None:
        out = torch.empty((B, H, N, d), dtype=torch.bfloat16, device=qc.device)
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
        out = torch.empty_like(q)
    st = lib().mxattn_cross_forward(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, H,
                                    Nq, Nkv, d, _mode(mode), _stream(stream))
    _check(st, "mxattn_cross_forward")
    return out


def cross_attend(qc, qs, kc, ks, vc, vs, Nq: int, Nkv: int, mode, out=None, stream=None):
    """The fused kernel on quantized operands with Nq queries and Nkv keys."""
    B, H = qc.shape[0], qc.shape[1]
    d = qc.shape[3] * 2
    if out is None:
        out = torch.empty((B, H, Nq, d), dtype=torch.bfloat16, device=qc.device)
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
        q_out = q.new_empty((B, Hq, N, d))
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
            k_out = q.new_empty((B, Hkv, N, d))
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


def _cache(k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len, index, d):
    """Checked addresses and sizes of a cache of d channels and its batch, as the library takes them, and the cache's
    heads."""
    if k_codes.dim() != 6 or page_table.dim() != 2:
        raise ValueError("k_codes must be [pages, heads, page_tokens / 32, 8, 32, 16], page_table [seqs, max_pages]")
    pages, heads, blocks, *block = k_codes.shape
    if block != [d // 16, BLOCK_TOKENS, 16] or v_codes.shape != (pages, heads, blocks, d, BLOCK_TOKENS):
        raise ValueError(f"k_codes and v_codes must have the shapes of cache_shapes for heads of {d} channels")
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
    dev = _index(q, "q")
    qp, qst = _token_rows(q, "q", dev)
    tokens, Hq, d = q.shape
    cache, heads = _cache(k_codes, k_scales, v_codes, v_scales, page_table, q_start, kv_len, dev, d)
    if out is None:
        out = q.new_empty((tokens, Hq, d))
    elif out.shape != q.shape:
        raise ValueError("out must have q's shape")
    op, ost = _token_rows(out, "out", dev)
    L, work, size = _lib or lib(), None, 0
    if stream is None:  # torch's memory belongs to the current stream, and to the graph that is captured on it
        size = L.mxattn_cache_attend_workspace(cache[5], *cache[9:], tokens, Hq, heads, max_q, max_kv)
        if size:
            work = torch.empty(size, dtype=torch.uint8, device=q.device)
    _run(L.mxattn_cache_attend, "mxattn_cache_attend", dev, stream,
         (qp, qst, *cache, tokens, Hq, heads, d, causal, max_q, max_kv, op, ost,
          work.data_ptr() if size else None, size))
    return out


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
