"""Int8 linear layers between float activations, with a scale for each token and each output channel.

Beside the paper's integer path, whose scales are fixed per tensor and dyadic: here rows are quantised as they come
(i8_quantize), products are taken back to floats in their epilogue (i8_linear), by expert too (i8_grouped_linear).  Like mx.py,
this only marshals arguments, through the same binding.
"""
from __future__ import annotations

import struct
from typing import NamedTuple

from . import IlwError, mx
from .mx import _act, _bind

__all__ = ["I8Tensor", "i8_empty", "i8_quantize", "i8_dequantize", "i8_linear", "i8_grouped_linear", "I8Experts"]

# ilw_i8_gemm_t, in its natural alignment
_GEMM = struct.Struct("@IPqPPqqPPPqiiiiiPq")


def gemm_struct(*fields) -> bytes:
    """An ilw_i8_gemm_t of the given fields (all but struct_size)."""
    return _GEMM.pack(_GEMM.size, *fields)


class I8Tensor(NamedTuple):
    """An int8 tensor [..., rows, k]: ``codes`` int8 [..., rows, k], whose rows start on 16-byte boundaries (i8_empty makes such), and
    ``scales`` float32 [..., rows]; its values are codes x scales."""

    codes: object
    scales: object


def i8_empty(rows: int, k: int, device="cuda") -> I8Tensor:
    """Room for ``rows`` rows of ``k`` values (uninitialised)."""
    import torch

    return I8Tensor(torch.empty((rows, -(-k // 16) * 16), dtype=torch.int8, device=device)[:, :k], torch.empty(rows, dtype=torch.float32, device=device))


def i8_quantize(X, gather=None, out: I8Tensor | None = None) -> I8Tensor:
    """ilwdetr_i8_quantize: X [rows, K] (float32, float16 or bfloat16), or its rows ``gather`` (int32; -1: a row of zeros), to int8
    with a scale each."""
    got = (mx._bound or _bind()).i8_quantize(X, gather, out)
    return I8Tensor(*got) if out is None else out


def i8_dequantize(m: I8Tensor, dtype=None, out=None):
    """ilwdetr_i8_dequantize: the values of an int8 matrix, in float32 unless ``dtype`` says otherwise."""
    return (mx._bound or _bind()).i8_dequantize(m, dtype, out)


def i8_linear(A: I8Tensor, W: I8Tensor, bias=None, act="none", out_dtype=None, out=None):
    """ilwdetr_i8_gemm: act(A W^T + bias) of int8 A [M, K] and W [N, K] -> [M, N] (bfloat16 unless ``out_dtype`` or ``out`` says
    otherwise).  ``act``: "none", "gelu", or "silu_gate" (rows of W alternate between gate and gated, see gate_rows; -> [M, N / 2])."""
    return (mx._bound or _bind()).i8_gemm(A, W, None, bias, _act(act), out_dtype, out)


def i8_grouped_linear(A: I8Tensor, W: I8Tensor, offsets, bias=None, act="none", out_dtype=None, out=None):
    """ilwdetr_i8_gemm by expert: rows offsets[e] .. offsets[e + 1] - 1 of A times W[e] (W [E, N, K], bias [E, N]; offsets int32
    [E + 1] on the device).  Rows of no expert are zero."""
    if offsets is None:
        raise IlwError("i8_grouped_linear: offsets are needed")
    return (mx._bound or _bind()).i8_gemm(A, W, offsets, bias, _act(act), out_dtype, out)


class I8Experts(mx.MxExperts):
    """MxExperts with int8 weights and activations: weights have a scale a channel, tokens and hidden rows one each."""

    quantize = staticmethod(i8_quantize)
    grouped_linear = staticmethod(i8_grouped_linear)

    @staticmethod
    def pack(w):
        E, N, K = w.shape
        q = i8_quantize(w.reshape(E * N, K))
        return I8Tensor(q.codes.unflatten(0, (E, N)), q.scales.view(E, N))
