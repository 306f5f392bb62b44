"""Microscaled 4-bit (MXFP4) linear layers and a mixture-of-experts feed-forward built from them.

As in the rest of the package, this only marshals arguments for ``libilwdetr.so``: torch tensors are device memory, calls
run on the current CUDA stream, and nothing is computed here.  The calls are short, so tensors are read and results
allocated in ``_mxbind.so`` (csrc/mx_bind.cpp), which raises ``IlwError`` like the rest.
"""
from __future__ import annotations

import ctypes
import os
import struct
from typing import NamedTuple

from . import IlwError, lib

__all__ = ["MxTensor", "Routing", "mx_empty", "mx_quantize", "mx_dequantize", "mx_linear", "mx_grouped_linear", "moe_route", "moe_combine",
           "gate_rows", "MxExperts"]

ACTS = {"none": 0, "gelu": 1, "silu_gate": 2}
SCORES = {"softmax": 0, "sigmoid": 1}
BIND_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_mxbind.so")

# ilw_mx_gemm_t, in its natural alignment
_GEMM = struct.Struct("@IPqPqPqqPqqPPqiiiiiPq")


def gemm_struct(*fields) -> bytes:
    """An ilw_mx_gemm_t of the given fields (all but struct_size)."""
    return _GEMM.pack(_GEMM.size, *fields)


class MxTensor(NamedTuple):
    """An MXFP4 tensor [..., rows, k]: ``codes`` uint8 [..., rows, 16 ceil(k / 32)], two E2M1 codes a byte with the lower
    nibble first, and ``scales`` uint8 [..., rows, >= ceil(k / 32)], one E8M0 byte for 32 consecutive values.  Rows start on
    16-byte boundaries; codes past k are zero."""

    codes: object
    scales: object
    k: int


class Routing(NamedTuple):
    """What ilwdetr_moe_route gives: expert and weight [T, k], offsets [E + 1], source [T k], slot [T, k]."""

    expert: object
    weight: object
    offsets: object
    source: object
    slot: object


_bound = None


def _bind():
    """_mxbind, holding the entry points of the loaded library."""
    global _bound
    if _bound is None:
        import torch  # noqa: F401  (its libraries are what the binding is linked with)

        L = lib()
        if not os.path.exists(BIND_PATH):
            raise IlwError(f"{BIND_PATH} is missing: build it with __graft_entry__.build()")
        try:
            from . import _mxbind
        except ImportError as e:  # (of another Python or torch)
            raise IlwError(f"{BIND_PATH} does not load, build it again with __graft_entry__.build(): {e}") from e

        names = ("ilwdetr_last_error", "ilwdetr_mx_quantize", "ilwdetr_mx_dequantize", "ilwdetr_mx_gemm", "ilwdetr_moe_route_workspace_bytes",
                 "ilwdetr_moe_route", "ilwdetr_moe_combine", "ilwdetr_moe_route_scored", "ilwdetr_i8_quantize", "ilwdetr_i8_dequantize", "ilwdetr_i8_gemm")
        _mxbind.bind(IlwError, *(ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in names))
        _bound = _mxbind
    return _bound


def mx_empty(rows: int, k: int, device="cuda") -> MxTensor:
    """Room for ``rows`` rows of ``k`` values (uninitialised)."""
    import torch

    nb = (k + 31) // 32
    return MxTensor(torch.empty((rows, 16 * nb), dtype=torch.uint8, device=device),
                    torch.empty((rows, -(-nb // 16) * 16), dtype=torch.uint8, device=device), k)


def mx_quantize(X, gather=None, out: MxTensor | None = None) -> MxTensor:
    """ilwdetr_mx_quantize: X [rows, K] (float32, float16, bfloat16 or int8), or its rows ``gather`` (int32; -1: a row of
    zeros), to MXFP4.  Rows of ``out``'s scales hold a multiple of 16 bytes, as mx_empty makes them: the call fills them up
    with zeros."""
    got = (_bound or _bind()).quantize(X, gather, out)
    return MxTensor(*got) if out is None else out


def mx_dequantize(m: MxTensor, dtype=None, out=None):
    """ilwdetr_mx_dequantize: the values of an MXFP4 matrix, in float32 unless ``dtype`` says otherwise."""
    return (_bound or _bind()).dequantize(m, dtype, out)


def _act(act) -> int:
    code = ACTS.get(act)
    if code is None:
        raise IlwError(f"act {act!r} is none of {', '.join(ACTS)}")
    return code


def mx_linear(A: MxTensor, W: MxTensor, bias=None, act="none", out_dtype=None, out=None):
    """ilwdetr_mx_gemm: act(A W^T + bias) of MXFP4 A [M, K] and W [N, K] -> [M, N] (bfloat16 unless ``out_dtype`` or ``out``
    says otherwise).  ``act``: "none", "gelu", or "silu_gate" (rows of W alternate between gate and gated, see gate_rows;
    -> [M, N / 2])."""
    return (_bound or _bind()).gemm(A, W, None, bias, _act(act), out_dtype, out)


def mx_grouped_linear(A: MxTensor, W: MxTensor, offsets, bias=None, act="none", out_dtype=None, out=None):
    """ilwdetr_mx_gemm by expert: rows offsets[e] .. offsets[e + 1] - 1 of A times W[e] (W [E, N, K], bias [E, N]; offsets int32
    [E + 1] on the device).  Rows of no expert are zero."""
    if offsets is None:
        raise IlwError("mx_grouped_linear: offsets are needed")
    return (_bound or _bind()).gemm(A, W, offsets, bias, _act(act), out_dtype, out)


def moe_route(logits, k: int, renormalize=True, score="softmax", bias=None, groups=1, top_groups=None, group_best=2, scale=1.0) -> Routing:
    """ilwdetr_moe_route: the k experts of each row of logits [T, E], their weights, and the rows' order by expert.

    ilwdetr_moe_route_scored, where anything after ``renormalize`` is given: experts are taken by their ``score`` ("softmax" or
    "sigmoid") plus ``bias`` (float32 [E], for balance: it chooses but does not weigh), among the ``top_groups`` (all) of ``groups``
    groups of consecutive experts that rank best by the sum of their ``group_best`` (1 or 2) largest; the weights are the scores, over
    their sum with ``renormalize``, times ``scale``."""
    bound = _bound or _bind()
    if score == "softmax" and bias is None and groups == 1 and scale == 1.0 and top_groups in (None, 1) and group_best in (1, 2):
        return Routing(*bound.route(logits, k, renormalize))
    code = SCORES.get(score)
    if code is None:
        raise IlwError(f"score {score!r} is none of {', '.join(SCORES)}")
    return Routing(*bound.route_scored(logits, k, renormalize, code, bias, groups, groups if top_groups is None else top_groups, group_best, scale))


def moe_combine(Y, slot, weight, residual=None, out=None):
    """ilwdetr_moe_combine: out[t] = (residual[t] +) sum_j weight[t, j] Y[slot[t, j]], in Y's type."""
    return (_bound or _bind()).combine(Y, slot, weight, residual, out)


def gate_rows(gate, up, dim=None):
    """Weight rows or biases of a gated layer in the order of ``act="silu_gate"``: gate_0, up_0, gate_1, up_1, ...  ``dim`` is
    the axis of the rows; unless given, that of weights [F, K] or [E, F, K] and of a bias [F].  Biases of experts [E, F] need
    ``dim=1``: nothing tells them from the weights of one layer."""
    import torch

    if dim is None:
        dim = 0 if gate.dim() < 3 else 1
    elif dim < 0:
        dim += gate.dim()
    return torch.stack([gate, up], dim + 1).flatten(dim, dim + 1)


class MxExperts:
    """A mixture-of-experts feed-forward on MXFP4 weights: route, gather and quantise the tokens by expert, first
    product with its activation, quantise, second product, weighted join onto the residual.

    ``w1`` [E, F1, d] and ``w2`` [E, d, F] are float CUDA tensors, quantised here once; with ``act`` "silu_gate" F1 = 2 F and
    the rows of w1 alternate (gate_rows), else F1 = F.  Biases are float32 [E, F1] (gated: gate_rows with dim=1) and [E, d].
    What follows ``renormalize`` is as in moe_route, which refuses here what it would refuse in forward."""

    def __init__(self, w1, w2, top: int, act="silu_gate", b1=None, b2=None, renormalize=True, *, score="softmax", bias=None, groups=1,
                 top_groups=None, group_best=2, scale=1.0):
        self.top, self.act, self.b1, self.b2, self.renormalize = top, act, b1, b2, renormalize
        self.routing = dict(score=score, bias=bias, groups=groups, top_groups=top_groups, group_best=group_best, scale=scale)
        moe_route(w1.new_empty((0, w1.shape[0])), top, renormalize, **self.routing)  # (of no tokens: its checks)
        self.w1, self.w2 = self.pack(w1), self.pack(w2)
        if w1.shape[0] != w2.shape[0] or w2.shape[2] * (2 if act == "silu_gate" else 1) != w1.shape[1] or w1.shape[2] != w2.shape[1]:
            raise IlwError(f"{type(self).__name__}: w1 {tuple(w1.shape)} and w2 {tuple(w2.shape)} do not follow one another")

    quantize = staticmethod(mx_quantize)
    grouped_linear = staticmethod(mx_grouped_linear)

    @staticmethod
    def pack(w):
        E, N, K = w.shape
        q = mx_quantize(w.reshape(E * N, K))
        return MxTensor(q.codes.view(E, N, -1), q.scales.view(E, N, -1), K)

    def forward(self, x, logits, residual=None):
        """x [T, d] and its router logits [T, E] -> [T, d] in x's type (plus ``residual``)."""
        r = moe_route(logits, self.top, self.renormalize, **self.routing)
        a = self.quantize(x, gather=r.source)
        h = self.grouped_linear(a, self.w1, r.offsets, bias=self.b1, act=self.act, out_dtype=x.dtype)
        y = self.grouped_linear(self.quantize(h), self.w2, r.offsets, bias=self.b2, out_dtype=x.dtype)
        return moe_combine(y, r.slot, r.weight, residual=residual)
