"""Thin Python binding of the low-bit part of libenec's C ABI (include/enec_lowbit.h).

Matrices in microscaled 4-bit floating point with the products that read them, and a paged 8-bit cache with its
attention.  As in enec.py: argument marshalling only, PyTorch for device memory and streams, status codes returned, no CPU
fallback.  The tensors' shapes, integer types and places are checked here, where C sees pointers only; a wrong one raises ValueError.
"""
from __future__ import annotations

import ctypes as C
import struct

from . import enec
from .enec import BF16, E_ARG, E_BLOCK, E_CAPACITY, E_DTYPE, FP16, FP32, OK, strerror  # noqa: F401

EXPORTS = ["enec_mx4_bytes", "enec_mx4_quantize", "enec_mx4_dequantize", "enec_mx4_linear_workspace", "enec_mx4_linear",
           "enec_mx4_matmul_workspace", "enec_mx4_matmul", "enec_cache_write", "enec_cache_read", "enec_cache_attention_workspace",
           "enec_cache_attention"]


class CacheStruct(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_scales", C.c_void_p), ("v_codes", C.c_void_p), ("v_scales", C.c_void_p),
                ("n_pages", C.c_uint32), ("page_tokens", C.c_uint32), ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32)]


class BatchStruct(C.Structure):
    _fields_ = [("table", C.c_void_p), ("starts", C.c_void_p), ("lengths", C.c_void_p), ("table_stride", C.c_uint32),
                ("batch", C.c_uint32), ("n_tokens", C.c_uint32), ("status", C.c_void_p)]


_lib = None


def lib():
    """libenec.so with this part's entry points declared."""
    global _lib
    if _lib is None:
        L = enec.lib()
        vp, sz, u32, i = C.c_void_p, C.c_size_t, C.c_uint32, C.c_int
        cache, batch = C.POINTER(CacheStruct), vp            # (a batch is handed over packed, see _BATCH)
        for name, result, arguments in (
                ("enec_mx4_bytes", i, [sz, sz, C.POINTER(sz), C.POINTER(sz)]),
                ("enec_mx4_quantize", i, [vp, sz, sz, sz, i, vp, vp, vp]),
                ("enec_mx4_dequantize", i, [vp, vp, sz, sz, vp, sz, i, vp]),
                ("enec_mx4_linear_workspace", sz, [sz, sz, sz]),
                ("enec_mx4_linear", i, [vp, sz, sz, i, vp, vp, sz, sz, vp, sz, vp, sz, vp]),
                ("enec_mx4_matmul_workspace", sz, [sz, sz, sz]),
                ("enec_mx4_matmul", i, [vp, vp, sz, vp, vp, sz, sz, vp, sz, i, vp, sz, vp]),
                ("enec_cache_write", i, [cache, batch, vp, sz, sz, vp, sz, sz, i, vp]),
                ("enec_cache_read", i, [cache, batch, vp, sz, sz, vp, sz, sz, i, vp]),
                ("enec_cache_attention_workspace", sz, [cache, u32, u32, u32, u32, u32]),
                ("enec_cache_attention", i, [cache, batch, vp, sz, sz, vp, sz, sz, i, u32, u32, u32, C.c_float, vp, sz, vp])):
            f = getattr(L, name)
            f.restype, f.argtypes = result, arguments
        _lib = L
    return _lib


_codes = None


def _dtype(t) -> int:
    """The library's code for a tensor's format; -1, which every call refuses, for any other."""
    global _codes
    if _codes is None:
        import torch
        _codes = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}
    return _codes.get(t.dtype, -1)


def _on_gpu(*tensors):
    """All of them (None: none) lie on one GPU, or in pinned host memory, which its kernels reach too.  (The calls compare the numbers of their tensors' GPUs
    themselves, 0.04 us each, and ask here where these differ.)"""
    device = -1
    for t in tensors:
        at = -1 if t is None else t.get_device()
        if at < 0:
            if t is not None and not t.is_pinned():
                raise ValueError("tensors on the GPU are wanted")
        elif device < 0:
            device = at
        elif at != device:
            raise ValueError("tensors on one GPU are wanted")


def _rows(t, what):
    """(rows, columns, row stride) of a matrix whose rows are runs."""
    shape = t.shape                                         # (an attribute of a tensor costs 0.1 us: each is asked for once)
    if len(shape) == 2:
        rows, cols = shape
        stride, side = t.stride()
        if side == 1 or cols <= 1:
            return rows, cols, stride if rows > 1 else cols
    raise ValueError(f"{what}: a matrix whose columns lie side by side is wanted")


def _mx4(codes, scales, what):
    """(rows, padded columns) of a matrix in 4 bits."""
    rows, half = codes.shape
    n, blocks = scales.shape
    if half & 63 or half != 16 * blocks or n != rows or codes.itemsize != 1 or scales.itemsize != 1 \
            or not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError(f"{what}: codes (rows, padded / 2) and scales (rows, padded / 32) of bytes without gaps are wanted, padded a multiple of 128")
    return rows, 2 * half


def _space(workspace):
    return (None, 0) if workspace is None else (workspace.data_ptr(), workspace.nbytes)


# ---- matrices in 4 bits -------------------------------------------------------------
def mx4_bytes(rows: int, cols: int) -> tuple:
    """(bytes of the codes, bytes of the scales) of a rows x cols matrix."""
    codes, scales = C.c_size_t(0), C.c_size_t(0)
    enec._check(lib().enec_mx4_bytes(rows, cols, C.byref(codes), C.byref(scales)), "enec_mx4_bytes")
    return codes.value, scales.value


def mx4_empty(rows: int, cols: int, device="cuda") -> tuple:
    """Tensors for a rows x cols matrix: codes (rows, padded / 2) and scales (rows, padded / 32), padded = cols up to a multiple of 128."""
    import torch
    padded = -(-cols // 128) * 128
    return (torch.empty(rows, padded // 2, dtype=torch.uint8, device=device), torch.empty(rows, padded // 32, dtype=torch.uint8, device=device))


def _same_padding(padded, cols):
    if not 0 <= padded - cols < 128:
        raise ValueError(f"{cols} columns are padded to {-(-cols // 128) * 128}, not {padded}")


def mx4_quantize(src, codes, scales, stream=None) -> int:
    """Enqueues enec_mx4_quantize.  src: (rows, cols) of bf16, fp16 or fp32; codes, scales: see mx4_empty."""
    rows, cols, stride = _rows(src, "src")
    n, padded = _mx4(codes, scales, "codes")
    _same_padding(padded, cols)
    if n != rows:
        raise ValueError("src and codes differ in their rows")
    if not src.get_device() == codes.get_device() == scales.get_device() >= 0:
        _on_gpu(src, codes, scales)
    return lib().enec_mx4_quantize(src.data_ptr(), rows, cols, stride, _dtype(src), codes.data_ptr(), scales.data_ptr(),
                                   enec._stream_handle(stream))


def mx4_dequantize(codes, scales, out, stream=None) -> int:
    """Enqueues enec_mx4_dequantize.  out: (rows, cols) of bf16, fp16 or fp32."""
    rows, cols, stride = _rows(out, "out")
    n, padded = _mx4(codes, scales, "codes")
    _same_padding(padded, cols)
    if n != rows:
        raise ValueError("out and codes differ in their rows")
    if not codes.get_device() == scales.get_device() == out.get_device() >= 0:
        _on_gpu(codes, scales, out)
    return lib().enec_mx4_dequantize(codes.data_ptr(), scales.data_ptr(), rows, cols, out.data_ptr(), stride, _dtype(out),
                                     enec._stream_handle(stream))


def mx4_linear_workspace(m: int, n: int, k: int) -> int:
    return int(lib().enec_mx4_linear_workspace(m, n, k))


def mx4_linear(x, codes, scales, out, workspace=None, stream=None) -> int:
    """Enqueues enec_mx4_linear: out (m, n) = x (m, k) w^T, x and out bf16 or fp16, w (n, k) in 4 bits."""
    m, k, x_stride = _rows(x, "x")
    n, padded = _mx4(codes, scales, "codes")
    _same_padding(padded, k)
    rows, cols, y_stride = _rows(out, "out")
    if (rows, cols) != (m, n) or out.dtype != x.dtype:
        raise ValueError(f"out: ({m}, {n}) of x's format is wanted")
    if not x.get_device() == codes.get_device() == scales.get_device() == out.get_device() == (x if workspace is None else workspace).get_device() >= 0:
        _on_gpu(x, codes, scales, out, workspace)
    ws, size = _space(workspace)
    return lib().enec_mx4_linear(x.data_ptr(), m, x_stride, _dtype(x), codes.data_ptr(), scales.data_ptr(), n, k, out.data_ptr(), y_stride,
                                 ws, size, enec._stream_handle(stream))


def mx4_matmul_workspace(m: int, n: int, k: int) -> int:
    return int(lib().enec_mx4_matmul_workspace(m, n, k))


def mx4_matmul(x_codes, x_scales, codes, scales, out, workspace=None, stream=None) -> int:
    """Enqueues enec_mx4_matmul: out (m, n) = x w^T with both in 4 bits; out bf16, fp16 or fp32."""
    m, padded = _mx4(x_codes, x_scales, "x_codes")
    n, other = _mx4(codes, scales, "codes")
    rows, cols, y_stride = _rows(out, "out")
    if padded != other or (rows, cols) != (m, n):
        raise ValueError(f"matrices of as many columns and out ({m}, {n}) are wanted")
    if not x_codes.get_device() == x_scales.get_device() == codes.get_device() == scales.get_device() == out.get_device() \
            == (out if workspace is None else workspace).get_device() >= 0:
        _on_gpu(x_codes, x_scales, codes, scales, out, workspace)
    ws, size = _space(workspace)
    return lib().enec_mx4_matmul(x_codes.data_ptr(), x_scales.data_ptr(), m, codes.data_ptr(), scales.data_ptr(), n, padded, out.data_ptr(),
                                 y_stride, _dtype(out), ws, size, enec._stream_handle(stream))


# ---- the cache ----------------------------------------------------------------------
class Cache:
    """Device tensors of a paged cache: k_codes (pages, heads, page_tokens, head_dim) and v_codes (pages, heads, head_dim, page_tokens) of
    E4M3 bytes, k_scales and v_scales (pages, heads) of exponent bytes."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        pages, heads, page, dim = k_codes.shape
        if tuple(v_codes.shape) != (pages, heads, dim, page) or tuple(k_scales.shape) != (pages, heads) or tuple(v_scales.shape) != (pages, heads):
            raise ValueError("k_codes (pages, heads, page_tokens, head_dim), v_codes (pages, heads, head_dim, page_tokens) and scales (pages, heads) are wanted")
        for t in (k_codes, k_scales, v_codes, v_scales):
            if t.element_size() != 1 or not t.is_contiguous():
                raise ValueError("the cache's tensors are bytes without gaps")
            if t.device != k_codes.device:
                raise ValueError("the cache's tensors are on one GPU")
        self.tensors = (k_codes, k_scales, v_codes, v_scales)
        self.device = k_codes.get_device()
        self.page_tokens, self.heads, self.head_dim, self.n_pages = page, heads, dim, pages
        self.struct = CacheStruct(*(t.data_ptr() for t in self.tensors), pages, page, heads, dim)
        self.ref = C.byref(self.struct)

    @classmethod
    def empty(cls, n_pages: int, heads: int, head_dim: int, page_tokens: int = 64, device="cuda"):
        """A cache of n_pages free pages (their contents do not matter: a page's first write sets its scale)."""
        import torch
        codes, scales = (n_pages, heads, page_tokens, head_dim), (n_pages, heads)
        make = lambda *shape: torch.empty(*shape, dtype=torch.uint8, device=device)  # noqa: E731
        return cls(make(*codes), make(*scales), make(n_pages, heads, head_dim, page_tokens), make(*scales))


_BATCH = struct.Struct("=QQQIII4xQ")          # a BatchStruct: packed in one go, a structure's fields cost 0.2 us each
assert _BATCH.size == C.sizeof(BatchStruct)


_int32 = None


def _batch(cache, x, y, table, starts, lengths, n_tokens, status, workspace=None):
    global _int32
    if _int32 is None:
        import torch
        _int32 = torch.int32
    shape = table.shape
    batch = lengths.numel()
    if len(shape) != 2 or shape[0] != batch or starts.numel() != batch + 1:
        raise ValueError("table (batch, pages) has a row for each of lengths, starts one entry more")
    if table.dtype is not _int32 or starts.dtype is not _int32 or lengths.dtype is not _int32 \
            or not table.is_contiguous() or not starts.is_contiguous() or not lengths.is_contiguous():
        raise ValueError("table, starts and lengths are int32 without gaps")
    if status is not None and (status.dtype is not _int32 or status.numel() == 0):
        raise ValueError("status: an int32 word, or None, is wanted")
    if not x.get_device() == y.get_device() == table.get_device() == starts.get_device() == lengths.get_device() == (x if status is None else status).get_device() \
            == (x if workspace is None else workspace).get_device() == cache.device >= 0:
        _on_gpu(cache.tensors[0], x, y, table, starts, lengths, status, workspace)
    return _BATCH.pack(table.data_ptr(), starts.data_ptr(), lengths.data_ptr(), shape[1], batch, n_tokens,
                       0 if status is None else status.data_ptr())


def _tokens(t, other, heads, dim, what):
    """(tokens, token stride, head stride, other's token stride, head stride) of two tensors of (tokens, heads, head_dim) values."""
    shape = t.shape
    if len(shape) != 3 or shape != other.shape or t.dtype != other.dtype:
        raise ValueError(f"{what} are two tensors of (tokens, heads, head_dim) values, alike in shape and format")
    tokens, h, d = shape
    token, head, side = t.stride()
    other_token, other_head, other_side = other.stride()
    if h != heads or d != dim or side != 1 or other_side != 1:
        raise ValueError(f"{what}: (tokens, {heads}, {dim}) values, a head's side by side, are wanted")
    return tokens, token, head, other_token, other_head


def cache_write(cache, k, v, table, starts, lengths, status=None, stream=None) -> int:
    """Enqueues enec_cache_write.  k, v: (tokens, heads, head_dim) of bf16 or fp16, the newest tokens of their sequences; table (batch,
    pages), starts (batch + 1) and lengths (batch, new tokens included): int32 on the device; status: None or an int32 word holding 0."""
    tokens, kt, kh, vt, vh = _tokens(k, v, cache.heads, cache.head_dim, "k and v")
    b = _batch(cache, k, v, table, starts, lengths, tokens, status)
    return lib().enec_cache_write(cache.ref, b, k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, _dtype(k), enec._stream_handle(stream))


def cache_read(cache, k, v, table, starts, lengths, status=None, stream=None) -> int:
    """Enqueues enec_cache_read: the newest tokens' keys and values into k, v (bf16, fp16 or fp32); starts of whole lengths read all."""
    tokens, kt, kh, vt, vh = _tokens(k, v, cache.heads, cache.head_dim, "k and v")
    b = _batch(cache, k, v, table, starts, lengths, tokens, status)
    return lib().enec_cache_read(cache.ref, b, k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, _dtype(k), enec._stream_handle(stream))


def cache_attention_workspace(cache, batch: int, n_tokens: int, q_heads: int, max_new: int, max_length: int) -> int:
    return int(lib().enec_cache_attention_workspace(cache.ref, batch, n_tokens, q_heads, max_new, max_length))


def cache_attention(cache, q, out, table, starts, lengths, max_new: int, max_length: int, workspace=None, scale: float | None = None,
                    status=None, stream=None) -> int:
    """Enqueues enec_cache_attention.  q, out: (tokens, q_heads, head_dim) of bf16 or fp16; scale: head_dim ** -0.5 unless given."""
    heads, dim = q.shape[1], cache.head_dim
    tokens, qt, qh, ot, oh = _tokens(q, out, heads, dim, "q and out")
    b = _batch(cache, q, out, table, starts, lengths, tokens, status, workspace)
    ws, size = _space(workspace)
    return lib().enec_cache_attention(cache.ref, b, q.data_ptr(), qt, qh, out.data_ptr(), ot, oh, _dtype(q), heads, max_new, max_length,
                                      dim ** -0.5 if scale is None else scale, ws, size, enec._stream_handle(stream))
