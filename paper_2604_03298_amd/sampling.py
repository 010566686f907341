"""Thin Python binding of the sampling part of libenec's C ABI (include/enec_sampling.h).

One token for each row of logits.  As in lowbit.py: argument marshalling only, PyTorch for device memory and streams, status codes returned,
no CPU fallback; the tensors' shapes, types and places are checked here, and a wrong one raises ValueError.
"""
from __future__ import annotations

import ctypes as C

from . import enec
from .enec import E_ARG, E_CAPACITY, E_DTYPE, OK, strerror  # noqa: F401
from .lowbit import _dtype, _on_gpu, _rows, _space, _stream_on

EXPORTS = ["enec_sample_workspace", "enec_sample"]


class SamplingStruct(C.Structure):
    _fields_ = [("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p), ("uniform", C.c_void_p)]


_lib = None


def lib():
    """libenec.so with this part's entry points declared."""
    global _lib
    if _lib is None:
        L = enec.lib()
        vp, sz, i = C.c_void_p, C.c_size_t, C.c_int
        L.enec_sample_workspace.restype, L.enec_sample_workspace.argtypes = sz, [sz, sz]
        L.enec_sample.restype, L.enec_sample.argtypes = i, [vp, sz, sz, sz, i, C.POINTER(SamplingStruct), vp, vp, vp, sz, vp]
        _lib = L
    return _lib


def sample_workspace(rows: int, vocab: int) -> int:
    return int(lib().enec_sample_workspace(rows, vocab))


def sample(logits, uniform, tokens, temperature=None, top_k=None, top_p=None, min_p=None, log_probs=None, workspace=None, stream=None) -> int:
    """Enqueues enec_sample.  logits: (rows, vocab) of bf16, fp16 or fp32; for each row: uniform, temperature, top_p and min_p fp32, top_k int32,
    each but uniform may be None; tokens: int32, log_probs: fp32 or None, for each row."""
    import torch
    rows, vocab, stride = _rows(logits, "logits")
    device = logits.get_device()
    at, there, others = [], [logits, workspace], device < 0 or (workspace is not None and workspace.get_device() != device)
    for t, kind, name in ((temperature, torch.float32, "temperature"), (top_k, torch.int32, "top_k"), (top_p, torch.float32, "top_p"),
                          (min_p, torch.float32, "min_p"), (uniform, torch.float32, "uniform"), (tokens, torch.int32, "tokens"),
                          (log_probs, torch.float32, "log_probs")):
        if t is None:
            at.append(None)
            continue
        if t.dtype is not kind or t.shape != (rows,) or not t.is_contiguous():
            raise ValueError(f"{name}: ({rows},) of {kind} without gaps is wanted")
        if t.get_device() != device:
            others = True
        there.append(t)
        at.append(t.data_ptr())
    if others:
        device = _on_gpu(*there)
    ws, size = _space(workspace)
    return lib().enec_sample(logits.data_ptr(), rows, vocab, stride, _dtype(logits), C.byref(SamplingStruct(*at[:5])), at[5], at[6], ws, size,
                             _stream_on(device, stream))
