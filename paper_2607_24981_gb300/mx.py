"""Microscaled 4-bit (MXFP4) linear layers and a mixture-of-experts feed-forward built from them.

As in the rest of the package, this only marshals arguments for ``libilwdetr.so``: torch tensors are device memory, calls
run on the current CUDA stream, and nothing is computed here.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple

from . import IlwError, _check, _ptr, _stream, lib

__all__ = ["MxTensor", "Routing", "mx_empty", "mx_quantize", "mx_dequantize", "mx_linear", "mx_grouped_linear", "moe_route", "moe_combine",
           "gate_rows", "MxExperts"]

FP32, FP16, BF16 = 232, 216, 217
ACTS = {"none": 0, "gelu": 1, "silu_gate": 2}


class MxGemmT(C.Structure):
    _fields_ = [
        ("struct_size", C.c_uint32),
        ("a_codes", C.c_void_p), ("a_ldc", C.c_int64), ("a_scales", C.c_void_p), ("a_lds", C.c_int64),
        ("w_codes", C.c_void_p), ("w_ldc", C.c_int64), ("w_codes_stride", C.c_int64),
        ("w_scales", C.c_void_p), ("w_lds", C.c_int64), ("w_scales_stride", C.c_int64),
        ("bias", C.c_void_p), ("offsets", C.c_void_p),
        ("M", C.c_int64), ("N", C.c_int32), ("K", C.c_int32), ("experts", C.c_int32), ("act", C.c_int32), ("y_form", C.c_int32),
        ("Y", C.c_void_p), ("ldy", C.c_int64),
    ]


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


def _form(dtype) -> int:
    import torch

    forms = {torch.float32: FP32, torch.float16: FP16, torch.bfloat16: BF16}
    if dtype not in forms:
        raise IlwError(f"{dtype} is neither float32, float16 nor bfloat16")
    return forms[dtype]


def _on(what, *tensors):
    """Device tensors whose last dimension is contiguous."""
    for t in tensors:
        if t is not None and (not t.is_cuda or (t.numel() and t.shape[-1] > 1 and t.stride(-1) != 1)):
            raise IlwError(f"{what}: a tensor is not on the GPU, or its last dimension is not contiguous")


def _row(t) -> int:
    """Elements between rows (no or a single row may carry any stride: then at least what holds a row)."""
    return t.stride(-2) if t.shape[-2] > 1 and t.numel() else max(t.stride(-2), t.shape[-1])


def _ints(what, *tensors):
    import torch

    for t in tensors:
        if t is not None and (t.dtype != torch.int32 or not t.is_contiguous() or not t.is_cuda):
            raise IlwError(f"{what}: indices, slots and offsets are contiguous int32 CUDA tensors")


def _parts(what, m: MxTensor, dims: int):
    import torch

    nb = (m.k + 31) // 32
    for t, width in ((m.codes, 16 * nb), (m.scales, nb)):
        if t.dtype != torch.uint8 or t.dim() != dims or t.shape[-1] < width or t.shape[:-1] != m.codes.shape[:-1]:
            raise IlwError(f"{what}: an MXFP4 tensor of k={m.k} has uint8 codes [..., {16 * nb}] and scales [..., >= {nb}] of {dims} dimensions")
    _on(what, m.codes, m.scales)


def mx_empty(rows: int, k: int, device="cuda") -> MxTensor:
    """Room for ``rows`` rows of ``k`` values (uninitialised)."""
    import torch

    nb = (k + 31) // 32
    return MxTensor(torch.empty((rows, 16 * nb), dtype=torch.uint8, device=device),
                    torch.empty((rows, -(-nb // 16) * 16), dtype=torch.uint8, device=device), k)


def mx_quantize(X, gather=None, out: MxTensor | None = None) -> MxTensor:
    """ilwdetr_mx_quantize: X [rows, K] (float32, float16, bfloat16 or int8), or its rows ``gather`` (int32; -1: a row of
    zeros), to MXFP4."""
    import torch

    if X.dim() != 2:
        raise IlwError(f"mx_quantize: X has {X.dim()} dimensions, not 2")
    _on("mx_quantize", X)
    _ints("mx_quantize", gather)
    form = 8 if X.dtype == torch.int8 else _form(X.dtype)
    rows, K = (X.shape[0] if gather is None else gather.numel()), X.shape[1]
    if out is None:
        out = mx_empty(rows, K, X.device)
    _parts("mx_quantize", out, 2)
    if out.k != K or out.codes.shape[0] != rows:
        raise IlwError(f"mx_quantize: out holds {out.codes.shape[0]} rows of {out.k}, not {rows} of {K}")
    _check(lib().ilwdetr_mx_quantize(_ptr(X), form, _row(X), X.shape[0], _ptr(gather), rows, K, _ptr(out.codes), _row(out.codes),
                                     _ptr(out.scales), _row(out.scales), _stream()), "mx_quantize")
    return out


def mx_dequantize(m: MxTensor, dtype=None, out=None):
    """ilwdetr_mx_dequantize: the values of an MXFP4 matrix, in float32 unless ``dtype`` says otherwise."""
    import torch

    _parts("mx_dequantize", m, 2)
    if out is None:
        out = torch.empty((m.codes.shape[0], m.k), dtype=dtype or torch.float32, device=m.codes.device)
    _on("mx_dequantize", out)
    if tuple(out.shape) != (m.codes.shape[0], m.k):
        raise IlwError(f"mx_dequantize: out is {tuple(out.shape)}, not {(m.codes.shape[0], m.k)}")
    _check(lib().ilwdetr_mx_dequantize(_ptr(m.codes), _row(m.codes), _ptr(m.scales), _row(m.scales), m.codes.shape[0], m.k,
                                       _ptr(out), _form(out.dtype), _row(out), _stream()), "mx_dequantize")
    return out


def _gemm(what, A, W, offsets, bias, act, out_dtype, out):
    import torch

    _parts(what, A, 2)
    _parts(what, W, 2 if offsets is None else 3)
    _ints(what, offsets)
    if act not in ACTS:
        raise IlwError(f"{what}: act {act!r} is none of {', '.join(ACTS)}")
    experts = 1 if offsets is None else W.codes.shape[0]
    M, N = A.codes.shape[0], W.codes.shape[-2]
    if A.k != W.k:
        raise IlwError(f"{what}: A has k={A.k}, W k={W.k}")
    if offsets is not None and offsets.numel() != experts + 1:
        raise IlwError(f"{what}: {experts} experts need {experts + 1} offsets, not {offsets.numel()}")
    if bias is not None and (bias.dtype != torch.float32 or not bias.is_contiguous() or not bias.is_cuda or bias.numel() != experts * N):
        raise IlwError(f"{what}: bias is a contiguous float32 tensor of {experts * N} values")
    wide = N // 2 if act == "silu_gate" else N
    if out is None:
        out = torch.empty((M, wide), dtype=out_dtype or torch.bfloat16, device=A.codes.device)
    _on(what, out)
    if tuple(out.shape) != (M, wide):
        raise IlwError(f"{what}: out is {tuple(out.shape)}, not {(M, wide)}")
    between = (lambda t: t.stride(0)) if offsets is not None else (lambda t: 0)
    desc = MxGemmT(C.sizeof(MxGemmT), A.codes.data_ptr(), _row(A.codes), A.scales.data_ptr(), _row(A.scales),
                   W.codes.data_ptr(), _row(W.codes), between(W.codes), W.scales.data_ptr(), _row(W.scales), between(W.scales),
                   None if bias is None else bias.data_ptr(), None if offsets is None else offsets.data_ptr(),
                   M, N, A.k, experts, ACTS[act], _form(out.dtype), out.data_ptr(), _row(out))
    _check(lib().ilwdetr_mx_gemm(C.byref(desc), _stream()), what)
    return out


def mx_linear(A: MxTensor, W: MxTensor, bias=None, act="none", out_dtype=None, out=None):
    """ilwdetr_mx_gemm: act(A W^T + bias) of MXFP4 A [M, K] and W [N, K] -> [M, N] (bfloat16 unless ``out_dtype`` or ``out``
    says otherwise).  ``act``: "none", "gelu", or "silu_gate" (rows of W alternate between gate and gated, see gate_rows;
    -> [M, N / 2])."""
    return _gemm("mx_linear", A, W, None, bias, act, out_dtype, out)


def mx_grouped_linear(A: MxTensor, W: MxTensor, offsets, bias=None, act="none", out_dtype=None, out=None):
    """ilwdetr_mx_gemm by expert: rows offsets[e] .. offsets[e + 1] - 1 of A times W[e] (W [E, N, K], bias [E, N]; offsets int32
    [E + 1] on the device).  Rows of no expert are zero."""
    return _gemm("mx_grouped_linear", A, W, offsets, bias, act, out_dtype, out)


def moe_route(logits, k: int, renormalize=True, workspace=None) -> Routing:
    """ilwdetr_moe_route: the k experts of each row of logits [T, E], their weights, and the rows' order by expert."""
    import torch

    if logits.dim() != 2:
        raise IlwError(f"moe_route: logits have {logits.dim()} dimensions, not 2")
    _on("moe_route", logits)
    T, E = logits.shape
    dev = logits.device
    need = int(lib().ilwdetr_moe_route_workspace_bytes(T, E))
    kk = max(k, 0)  # (the entry point refuses k < 1)
    i32 = torch.empty(3 * T * kk + E + 1, dtype=torch.int32, device=dev)
    expert, source, slot, offsets = i32.split([T * kk, T * kk, T * kk, E + 1])
    r = Routing(expert.view(T, kk), torch.empty((T, kk), dtype=torch.float32, device=dev), offsets, source, slot.view(T, kk))
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    _check(lib().ilwdetr_moe_route(_ptr(logits), _form(logits.dtype), _row(logits), T, E, k, int(bool(renormalize)), _ptr(r.expert),
                                   _ptr(r.weight), _ptr(r.offsets), _ptr(r.source), _ptr(r.slot), _ptr(workspace),
                                   workspace.numel() * workspace.element_size(), _stream()), "moe_route")
    return r


def moe_combine(Y, slot, weight, residual=None, out=None):
    """ilwdetr_moe_combine: out[t] = (residual[t] +) sum_j weight[t, j] Y[slot[t, j]], in Y's type."""
    import torch

    _on("moe_combine", Y, residual, out)
    _ints("moe_combine", slot)
    T, k = slot.shape
    if weight.dtype != torch.float32 or not weight.is_contiguous() or not weight.is_cuda or tuple(weight.shape) != (T, k):
        raise IlwError(f"moe_combine: weight is a contiguous float32 tensor {(T, k)}")
    N = Y.shape[1]
    if out is None:
        out = torch.empty((T, N), dtype=Y.dtype, device=Y.device)
    for t in (residual, out):
        if t is not None and (t.dtype != Y.dtype or tuple(t.shape) != (T, N)):
            raise IlwError(f"moe_combine: residual and out are {Y.dtype} {(T, N)}")
    _check(lib().ilwdetr_moe_combine(_ptr(Y), _form(Y.dtype), _row(Y), Y.shape[0], _ptr(slot), _ptr(weight), T, k, N, _ptr(residual),
                                     0 if residual is None else _row(residual), _ptr(out), _row(out), _stream()), "moe_combine")
    return out


def gate_rows(gate, up):
    """Weight rows (or biases) of a gated layer in the order of ``act="silu_gate"``: gate_0, up_0, gate_1, up_1, ..."""
    import torch

    dim = 0 if gate.dim() < 3 else 1
    return torch.stack([gate, up], dim + 1).flatten(dim, dim + 1)


class MxExperts:
    """A mixture-of-experts feed-forward on MXFP4 weights: route, gather and quantise the tokens by expert, first
    product with its activation, quantise, second product, weighted join onto the residual.

    ``w1`` [E, F1, d] and ``w2`` [E, d, F] are float CUDA tensors, quantised here once; with ``act`` "silu_gate" F1 = 2 F and
    the rows of w1 alternate (gate_rows), else F1 = F.  Biases are float32 [E, F1] and [E, d]."""

    def __init__(self, w1, w2, top: int, act="silu_gate", b1=None, b2=None, renormalize=True):
        self.top, self.act, self.b1, self.b2, self.renormalize = top, act, b1, b2, renormalize

        def pack(w):
            E, N, K = w.shape
            q = mx_quantize(w.reshape(E * N, K))
            return MxTensor(q.codes.view(E, N, -1), q.scales.view(E, N, -1), K)

        self.w1, self.w2 = pack(w1), pack(w2)
        if w1.shape[0] != w2.shape[0] or w2.shape[2] * (2 if act == "silu_gate" else 1) != w1.shape[1] or w1.shape[2] != w2.shape[1]:
            raise IlwError(f"MxExperts: w1 {tuple(w1.shape)} and w2 {tuple(w2.shape)} do not follow one another")

    def forward(self, x, logits, residual=None):
        """x [T, d] and its router logits [T, E] -> [T, d] in x's type (plus ``residual``)."""
        r = moe_route(logits, self.top, self.renormalize)
        a = mx_quantize(x, gather=r.source)
        h = mx_grouped_linear(a, self.w1, r.offsets, bias=self.b1, act=self.act, out_dtype=x.dtype)
        y = mx_grouped_linear(mx_quantize(h), self.w2, r.offsets, bias=self.b2, out_dtype=x.dtype)
        return moe_combine(y, r.slot, r.weight, residual=residual)
