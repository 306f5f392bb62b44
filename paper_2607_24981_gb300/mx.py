"""Microscaled 4-bit (MXFP4) linear layers and a mixture-of-experts feed-forward built from them.

As in the rest of the package, this only marshals arguments for ``libilwdetr.so``: torch tensors are device memory, calls
run on the current CUDA stream, and nothing is computed here.
"""
from __future__ import annotations

import struct
from typing import NamedTuple

from . import IlwError, _check, lib

__all__ = ["MxTensor", "Routing", "mx_empty", "mx_quantize", "mx_dequantize", "mx_linear", "mx_grouped_linear", "moe_route", "moe_combine",
           "gate_rows", "MxExperts"]

FP32, FP16, BF16 = 232, 216, 217
ACTS = {"none": 0, "gelu": 1, "silu_gate": 2}


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


# Calls of a few microseconds are common here, so each tensor's properties are read once, and torch's types are
# looked up once (on first use: the package itself imports without torch).
_T = None


class _Torch:
    def __init__(self):
        import torch

        self.torch, self.empty = torch, torch.empty
        self.u8, self.i32, self.f32, self.bf16 = torch.uint8, torch.int32, torch.float32, torch.bfloat16
        self.form = {torch.float32: FP32, torch.float16: FP16, torch.bfloat16: BF16}
        self.form_i8 = {**self.form, torch.int8: 8}
        self.stream = torch._C._cuda_getCurrentRawStream


def _torch() -> _Torch:
    global _T
    if _T is None:
        _T = _Torch()
    return _T


def _float(T, what, t, forms=None):
    """(form, rows, columns, elements between rows) of a float matrix on the GPU with contiguous rows.  No or a single row may
    carry any stride: then at least what holds a row."""
    form, shape, stride = (forms or T.form).get(t.dtype), t.shape, t.stride()
    if form is None:
        raise IlwError(f"{what}: {t.dtype} is none of {', '.join(str(d) for d in forms or T.form)}")
    if len(shape) != 2:
        raise IlwError(f"{what}: a tensor of {len(shape)} dimensions, not 2")
    rows, cols = shape
    if not t.is_cuda or (stride[1] != 1 and cols > 1 and rows > 0):
        raise IlwError(f"{what}: a tensor is not on the GPU, or its rows are not contiguous")
    return form, rows, cols, stride[0] if rows > 1 and cols > 0 else max(stride[0], cols)


def _index(T, what, t):
    if t.dtype is not T.i32 or not t.is_cuda or not t.is_contiguous():
        raise IlwError(f"{what}: indices, slots and offsets are contiguous int32 CUDA tensors")
    return t.data_ptr()


def _weights(T, what, name, t, n):
    if t.dtype is not T.f32 or not t.is_cuda or not t.is_contiguous() or t.numel() != n:
        raise IlwError(f"{what}: {name} is a contiguous float32 CUDA tensor of {n} values")
    return t.data_ptr()


def _parts(T, what, m, dims):
    """(shape, strides of codes, strides of scales) of an MXFP4 tensor."""
    codes, scales, k = m
    cs, ss, c, s = codes.shape, scales.shape, codes.stride(), scales.stride()
    nb = (k + 31) >> 5
    if codes.dtype is not T.u8 or scales.dtype is not T.u8 or len(cs) != dims or cs[-1] < 16 * nb or ss[-1] < nb or cs[:-1] != ss[:-1]:
        raise IlwError(f"{what}: an MXFP4 tensor of k={k} has uint8 codes [..., {16 * nb}] and scales [..., >= {nb}] of {dims} dimensions")
    if not codes.is_cuda or not scales.is_cuda or ((c[-1] != 1 or s[-1] != 1) and codes.numel()):
        raise IlwError(f"{what}: codes or scales are not on the GPU, or their rows are not contiguous")
    if cs[-2] <= 1 or not cs[-1]:  # (no or a single row may carry any stride)
        c, s = (*c[:-2], max(c[-2], 16 * (-cs[-1] // -16)), 1), (*s[:-2], max(s[-2], 16 * (-ss[-1] // -16)), 1)
    return cs, c, s


def mx_empty(rows: int, k: int, device="cuda") -> MxTensor:
    """Room for ``rows`` rows of ``k`` values (uninitialised)."""
    T = _torch()
    nb = (k + 31) >> 5
    return MxTensor(T.empty((rows, 16 * nb), dtype=T.u8, device=device), T.empty((rows, (nb + 15) & ~15), dtype=T.u8, device=device), k)


def mx_quantize(X, gather=None, out: MxTensor | None = None) -> MxTensor:
    """ilwdetr_mx_quantize: X [rows, K] (float32, float16, bfloat16 or int8), or its rows ``gather`` (int32; -1: a row of
    zeros), to MXFP4."""
    T = _torch()
    form, x_rows, K, ldx = _float(T, "mx_quantize", X, T.form_i8)
    rows, at = x_rows, None
    if gather is not None:
        rows, at = gather.numel(), _index(T, "mx_quantize", gather)
    if out is None:
        out = mx_empty(rows, K, X.device)
        nb = (K + 31) >> 5
        ldc, lds = 16 * nb, (nb + 15) & ~15
    else:
        shape, c, s = _parts(T, "mx_quantize", out, 2)
        ldc, lds = c[0], s[0]
        if out.k != K or shape[0] != rows:
            raise IlwError(f"mx_quantize: out holds {shape[0]} rows of {out.k}, not {rows} of {K}")
    _check(lib().ilwdetr_mx_quantize(X.data_ptr(), form, ldx, x_rows, at, rows, K, out.codes.data_ptr(), ldc, out.scales.data_ptr(), lds,
                                     T.stream(X.get_device())), "mx_quantize")
    return out


def mx_dequantize(m: MxTensor, dtype=None, out=None):
    """ilwdetr_mx_dequantize: the values of an MXFP4 matrix, in float32 unless ``dtype`` says otherwise."""
    T = _torch()
    shape, c, s = _parts(T, "mx_dequantize", m, 2)
    codes, scales, k = m
    rows = shape[0]
    if out is None:
        out = T.empty((rows, k), dtype=dtype or T.f32, device=codes.device)
    form, r, n, ldy = _float(T, "mx_dequantize", out)
    if r != rows or n != k:
        raise IlwError(f"mx_dequantize: out is {(r, n)}, not {(rows, k)}")
    _check(lib().ilwdetr_mx_dequantize(codes.data_ptr(), c[0], scales.data_ptr(), s[0], rows, k, out.data_ptr(), form, ldy,
                                       T.stream(codes.get_device())), "mx_dequantize")
    return out


def _gemm(what, A, W, offsets, bias, act, out_dtype, out):
    T = _torch()
    (M, _), ac, as_ = _parts(T, what, A, 2)
    code = ACTS.get(act)
    if code is None:
        raise IlwError(f"{what}: act {act!r} is none of {', '.join(ACTS)}")
    if offsets is None:
        (N, _), wc, ws = _parts(T, what, W, 2)
        experts, off, between = 1, None, (0, 0)
    else:
        (experts, N, _), wc, ws = _parts(T, what, W, 3)
        off, between = _index(T, what, offsets), (wc[0], ws[0])
        if offsets.numel() != experts + 1:
            raise IlwError(f"{what}: {experts} experts need {experts + 1} offsets, not {offsets.numel()}")
    if A.k != W.k:
        raise IlwError(f"{what}: A has k={A.k}, W k={W.k}")
    wide = N // 2 if code == 2 else N
    device = A.codes.get_device()
    if out is None:
        out = T.empty((M, wide), dtype=out_dtype or T.bf16, device=A.codes.device)
    form, r, n, ldy = _float(T, what, out)
    if r != M or n != wide:
        raise IlwError(f"{what}: out is {(r, n)}, not {(M, wide)}")
    desc = gemm_struct(A.codes.data_ptr(), ac[0], A.scales.data_ptr(), as_[0], W.codes.data_ptr(), wc[-2], between[0], W.scales.data_ptr(),
                       ws[-2], between[1], 0 if bias is None else _weights(T, what, "bias", bias, experts * N), off or 0, M, N, A.k, experts,
                       code, form, out.data_ptr(), ldy)
    _check(lib().ilwdetr_mx_gemm(desc, T.stream(device)), what)
    return out


def mx_linear(A: MxTensor, W: MxTensor, bias=None, act="none", out_dtype=None, out=None):
    """ilwdetr_mx_gemm: act(A W^T + bias) of MXFP4 A [M, K] and W [N, K] -> [M, N] (bfloat16 unless ``out_dtype`` or ``out``
    says otherwise).  ``act``: "none", "gelu", or "silu_gate" (rows of W alternate between gate and gated, see gate_rows;
    -> [M, N / 2])."""
    return _gemm("mx_linear", A, W, None, bias, act, out_dtype, out)


def mx_grouped_linear(A: MxTensor, W: MxTensor, offsets, bias=None, act="none", out_dtype=None, out=None):
    """ilwdetr_mx_gemm by expert: rows offsets[e] .. offsets[e + 1] - 1 of A times W[e] (W [E, N, K], bias [E, N]; offsets int32
    [E + 1] on the device).  Rows of no expert are zero."""
    if offsets is None:
        raise IlwError("mx_grouped_linear: offsets are needed")
    return _gemm("mx_grouped_linear", A, W, offsets, bias, act, out_dtype, out)


def moe_route(logits, k: int, renormalize=True) -> Routing:
    """ilwdetr_moe_route: the k experts of each row of logits [T, E], their weights, and the rows' order by expert."""
    t = _torch()
    form, T, E, ld = _float(t, "moe_route", logits)
    dev, L = logits.device, lib()
    kk = max(k, 0)  # (the entry point refuses k < 1)
    need = L.ilwdetr_moe_route_workspace_bytes(T, E)
    expert, slot = t.empty((T, kk), dtype=t.i32, device=dev), t.empty((T, kk), dtype=t.i32, device=dev)
    source, offsets = t.empty((T * kk,), dtype=t.i32, device=dev), t.empty((E + 1,), dtype=t.i32, device=dev)
    weight = t.empty((T, kk), dtype=t.f32, device=dev)
    workspace = t.empty((need,), dtype=t.u8, device=dev) if need else None
    _check(L.ilwdetr_moe_route(logits.data_ptr(), form, ld, T, E, k, 1 if renormalize else 0, expert.data_ptr(), weight.data_ptr(),
                               offsets.data_ptr(), source.data_ptr(), slot.data_ptr(), workspace.data_ptr() if need else None, need,
                               t.stream(logits.get_device())), "moe_route")
    return Routing(expert, weight, offsets, source, slot)


def moe_combine(Y, slot, weight, residual=None, out=None):
    """ilwdetr_moe_combine: out[t] = (residual[t] +) sum_j weight[t, j] Y[slot[t, j]], in Y's type."""
    t = _torch()
    form, rows, N, ldy = _float(t, "moe_combine", Y)
    at = _index(t, "moe_combine", slot)
    T, k = slot.shape
    w = _weights(t, "moe_combine", "weight", weight, T * k)
    if out is None:
        out, ldo = t.empty((T, N), dtype=Y.dtype, device=Y.device), N
    else:
        f, r, n, ldo = _float(t, "moe_combine", out)
        if (f, r, n) != (form, T, N):
            raise IlwError(f"moe_combine: out is {out.dtype} {(r, n)}, not {Y.dtype} {(T, N)}")
    res, ldr = None, 0
    if residual is not None:
        f, r, n, ldr = _float(t, "moe_combine", residual)
        res = residual.data_ptr()
        if (f, r, n) != (form, T, N):
            raise IlwError(f"moe_combine: residual is {residual.dtype} {(r, n)}, not {Y.dtype} {(T, N)}")
    _check(lib().ilwdetr_moe_combine(Y.data_ptr(), form, ldy, rows, at, w, T, k, N, res, ldr, out.data_ptr(), ldo,
                                     t.stream(Y.get_device())), "moe_combine")
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
