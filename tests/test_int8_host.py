"""Argument checks of the int8 entry points and of routing by scores: validate-only mode, so no kernel runs and the addresses
are never used; checks of the binding on tensors that have no memory."""
import ctypes
import struct

import pytest

from test_mx_host import L, on_gpu, refused  # noqa: F401  (L is the fixture of the library in validate-only mode)

V = ctypes.c_void_p(0x100000)


def test_quantize_checks(L):  # noqa: F811
    def q(X=V, form=232, ldx=100, x_rows=8, gather=None, rows=8, K=100, codes=V, ldc=112, scales=V):
        return L.ilwdetr_i8_quantize(X, form, ldx, x_rows, gather, rows, K, codes, ldc, scales, None)

    assert q() == 0 and q(form=216) == 0 and q(form=217, gather=V, rows=50) == 0 and q(ldc=1600) == 0
    assert q(rows=0, X=None, codes=None, scales=None) == 0
    assert q(X=None, x_rows=0, gather=V) == 0  # every index is then outside: rows of zeros
    refused(L, q(form=8), -1, b"x_form")
    refused(L, q(K=0), -1, b"sizes")
    refused(L, q(K=2**31 - 1, ldx=2**31), -1, b"sizes")
    refused(L, q(ldx=99), -1, b"sizes")
    refused(L, q(rows=9), -1, b"sizes")
    refused(L, q(X=None), -1, b"NULL")
    refused(L, q(X=ctypes.c_void_p(0x100002)), -1, b"misaligned")
    refused(L, q(gather=ctypes.c_void_p(0x100002)), -1, b"misaligned")
    refused(L, q(codes=ctypes.c_void_p(0x100008)), -1, b"codes")
    refused(L, q(ldc=96), -1, b"apart")
    refused(L, q(ldc=104), -1, b"apart")
    refused(L, q(scales=None), -1, b"scales")


def test_dequantize_checks(L):  # noqa: F811
    def d(codes=V, ldc=112, scales=V, rows=8, K=100, Y=V, form=217, ldy=100):
        return L.ilwdetr_i8_dequantize(codes, ldc, scales, rows, K, Y, form, ldy, None)

    assert d() == 0 and d(rows=0, codes=None, scales=None, Y=None) == 0
    refused(L, d(form=8), -1, b"y_form")
    refused(L, d(ldy=99), -1, b"sizes")
    refused(L, d(Y=ctypes.c_void_p(0x100001)), -1, b"Y")
    refused(L, d(codes=None), -1, b"codes")
    refused(L, d(ldc=100), -1, b"apart")


def test_product_checks(L):  # noqa: F811
    from paper_2607_24981_gb300 import int8

    fields = dict(a_codes=0x100000, a_ldc=256, a_scales=0x200000, w_codes=0x300000, w_ldc=256, w_codes_stride=256 * 64, w_scales=0x400000,
                  bias=0, offsets=0, M=300, N=64, K=250, experts=1, act=0, y_form=217, Y=0x500000, ldy=64)

    def g(**over):
        return L.ilwdetr_i8_gemm(int8.gemm_struct(*{**fields, **over}.values()), None)

    assert g() == 0 and g(M=0, Y=0, a_codes=0) == 0 and g(N=0) == 0
    assert g(offsets=0x600000, experts=5, bias=0x700000) == 0
    assert g(act=2, ldy=32) == 0  # a gated result has half the columns
    assert g(w_codes_stride=7) == 0  # one matrix: not read
    refused(L, L.ilwdetr_i8_gemm(bytes(200), None), -1, b"struct_size")
    refused(L, L.ilwdetr_i8_gemm(None, None), -1, b"struct_size")
    refused(L, g(act=3), -1, b"act")
    refused(L, g(y_form=8), -1, b"y_form")
    refused(L, g(K=0), -1, b"sizes")
    refused(L, g(M=-1), -1, b"sizes")
    refused(L, g(experts=2), -1, b"sizes")  # several experts need offsets
    refused(L, g(act=2, N=63), -1, b"even")
    refused(L, g(offsets=0x600000, experts=1025), -2, b"experts")
    refused(L, g(K=1 << 17, a_ldc=1 << 17, w_ldc=1 << 17), -2, b"2^17")  # sums of 2^14 each fit 32 bits below
    refused(L, g(M=(1 << 31) - 2048, N=1 << 20, ldy=1 << 20), -2, b"too large")
    refused(L, g(a_codes=0x100008), -1, b"A")
    refused(L, g(a_ldc=240), -1, b"A")
    refused(L, g(a_scales=0), -1, b"scales of A")
    refused(L, g(w_scales=0x400002), -1, b"scales of W")
    refused(L, g(w_ldc=250), -1, b"W")
    refused(L, g(offsets=0x600000, experts=5, w_codes_stride=0), -1, b"stride")
    refused(L, g(offsets=0x600000, experts=5, w_codes_stride=1032), -1, b"stride")
    refused(L, g(offsets=0x600002, experts=5), -1, b"misaligned")
    refused(L, g(ldy=63), -1, b"Y")
    refused(L, g(Y=0x500001), -1, b"Y")


def test_form_checks(L):  # noqa: F811
    from paper_2607_24981_gb300 import int8

    def f(M, N, K, experts=0, sms=152, out=True):
        got, ld = (ctypes.c_int32 * 3)(), -(-K // 16) * 16
        p = int8.gemm_struct(0x100000, ld, 0x200000, 0x300000, ld, N * ld, 0x400000, 0, 0x600000 if experts else 0, M, N, K, experts or 1, 0, 217, 0x500000, N)
        rc = L.ilwdetr_debug_i8_form(p, sms, got if out else None)
        return rc if rc else tuple(got)

    assert f(1, 4096, 4096) == (3, 1, 8) and f(8192, 8192, 8192) == (2, 1, 192)
    assert f(64, 4096, 4096)[:2] == (1, 4) and f(32, 4096, 2048, 64)[0] == 3
    for M in (1, 7, 100, 3000, 1 << 20):
        for N in (1, 130, 5000):
            for K in (1, 129, 9000, (1 << 17) - 1):
                for experts in (0, 1, 13, 1024):
                    got = f(M, N, K, experts)
                    assert got[0] in (0, 1, 2, 3) and got[1] in (1, 2, 4, 8) and 8 <= got[2] <= 192
    refused(L, f(0, 10, 10), -1, b"empty")
    refused(L, f(10, 10, 10, out=False), -1, b"NULL")
    refused(L, f(10, 10, 10, sms=-1), -1, b"sms")


def scores(size=None, score=1, groups=8, top_groups=4, group_best=2, scale=1.0, bias=0x100000):
    """An ilw_moe_scores_t."""
    s = struct.Struct("@IiiiifP")
    return s.pack(s.size if size is None else size, score, groups, top_groups, group_best, scale, bias)


def test_routing_by_scores_checks(L):  # noqa: F811
    def r(logits=V, form=217, ld=64, T=5000, E=64, k=4, offsets=V, slot=V, ws=V, size=1 << 20, q=None, **over):
        return L.ilwdetr_moe_route_scored(logits, form, ld, T, E, k, 1, scores(**over) if q is None else q, V, V, offsets, V, slot, ws, size, None)

    assert r() == 0 and r(T=0, logits=None, slot=None) == 0 and r(bias=0) == 0 and r(score=0, group_best=1) == 0
    assert r(T=16, ws=None, size=0) == 0
    assert r(groups=1, top_groups=1, k=16) == 0 and r(groups=32, top_groups=32) == 0
    refused(L, r(q=bytes(64)), -1, b"struct_size")
    refused(L, L.ilwdetr_moe_route_scored(V, 217, 64, 16, 64, 4, 1, None, V, V, V, V, V, V, 0, None), -1, b"scores")
    refused(L, r(score=2), -1, b"score")
    refused(L, r(groups=0), -1, b"groups")
    refused(L, r(groups=7), -1, b"groups")  # does not divide 64
    refused(L, r(top_groups=0), -1, b"groups")
    refused(L, r(top_groups=9), -1, b"groups")
    refused(L, r(group_best=3), -1, b"group_best")
    refused(L, r(groups=64), -2, b"groups")
    refused(L, r(top_groups=1, k=9), -1, b"k=9")  # a group has 8
    refused(L, r(scale=float("nan")), -1, b"scale")
    refused(L, r(scale=float("inf")), -1, b"scale")
    refused(L, r(bias=0x100002), -1, b"bias")
    refused(L, r(form=8), -1, b"form")
    refused(L, r(k=65), -1, b"sizes")
    refused(L, r(slot=None), -1, b"NULL")
    refused(L, r(size=16), -1, b"workspace")


def test_binding_refuses_what_it_cannot_pass_on():
    """Checks of the binding itself, on CPU tensors: none reaches the library."""
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    x = torch.zeros(4, 64)
    m = ilw.I8Tensor(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4))
    for call in (lambda: ilw.i8_quantize(x), lambda: ilw.i8_dequantize(m), lambda: ilw.i8_linear(m, m), lambda: ilw.moe_route(x, 2, score="sigmoid")):
        with pytest.raises(ilw.IlwError, match="GPU|CUDA"):
            call()
    with pytest.raises(ilw.IlwError, match="dimensions, not 2"):
        ilw.i8_quantize(torch.zeros(2, 2, 2))
    with pytest.raises(ilw.IlwError, match="float32, float16, bfloat16"):
        ilw.i8_quantize(torch.zeros(2, 2, dtype=torch.int8))
    with pytest.raises(ilw.IlwError, match="I8Tensor"):
        ilw.i8_linear(torch.zeros(2), m)
    with pytest.raises(ilw.IlwError, match="int8 tensor"):
        ilw.i8_grouped_linear(i8(4, 64), ilw.I8Tensor(m.codes[None], m.scales), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ilw.IlwError, match="offsets"):
        ilw.i8_grouped_linear(m, m, None)
    with pytest.raises(ilw.IlwError, match="act"):
        ilw.i8_linear(m, m, act="relu")
    with pytest.raises(ilw.IlwError, match="score"):
        ilw.moe_route(x, 2, score="tanh")


def i8(*shape, at="cuda:0", scales_at=None, scales=None, strides=None):
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    return ilw.I8Tensor(on_gpu(shape, torch.int8, at, strides=strides), on_gpu(shape[:-1] if scales is None else scales, torch.float32, scales_at or at))


def test_int8_tensors_that_do_not_fit_are_refused():
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    f = torch.float32
    for call in (lambda: ilw.i8_linear(i8(4, 64), i8(8, 80)), lambda: ilw.i8_linear(i8(4, 64, scales=(5,)), i8(8, 64)),
                 lambda: ilw.i8_linear(i8(4, 64, strides=(1, 4)), i8(8, 64)), lambda: ilw.i8_linear(i8(4, 0), i8(8, 0)),
                 lambda: ilw.i8_linear(i8(4, 64), i8(8, 64), out=on_gpu((4, 7), f)),
                 lambda: ilw.i8_linear(i8(4, 64), i8(8, 64), bias=on_gpu((2, 4), f)),
                 lambda: ilw.i8_grouped_linear(i8(4, 64), i8(3, 8, 64), on_gpu((3,), torch.int32)),
                 lambda: ilw.i8_quantize(on_gpu((4, 64), f), out=i8(4, 80)), lambda: ilw.i8_quantize(on_gpu((4, 64), f), out=i8(5, 64)),
                 lambda: ilw.i8_dequantize(i8(4, 64), out=on_gpu((4, 63), f)),
                 lambda: ilw.moe_route(on_gpu((4, 64), f), 2, bias=on_gpu((63,), f)), lambda: ilw.moe_route(on_gpu((4, 64), f), 2, bias=on_gpu((64,), torch.float16))):
        with pytest.raises(ilw.IlwError):
            call()


def test_tensors_of_more_than_one_gpu_are_refused():
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    far, i32, f = "cuda:1", torch.int32, torch.float32
    for call in (lambda: ilw.i8_quantize(on_gpu((4, 64), f), gather=on_gpu((4,), i32, far)), lambda: ilw.i8_quantize(on_gpu((4, 64), f), out=i8(4, 64, at=far)),
                 lambda: ilw.i8_dequantize(i8(4, 64, scales_at=far)), lambda: ilw.i8_dequantize(i8(4, 64), out=on_gpu((4, 64), f, far)),
                 lambda: ilw.i8_linear(i8(4, 64), i8(8, 64, at=far)), lambda: ilw.i8_linear(i8(4, 64), i8(8, 64, scales_at=far)),
                 lambda: ilw.i8_linear(i8(4, 64), i8(8, 64), bias=on_gpu((8,), f, far)), lambda: ilw.i8_linear(i8(4, 64), i8(8, 64), out=on_gpu((4, 8), f, far)),
                 lambda: ilw.i8_grouped_linear(i8(4, 64), i8(2, 8, 64), on_gpu((3,), i32, far)),
                 lambda: ilw.moe_route(on_gpu((4, 64), f), 2, bias=on_gpu((64,), f, far))):
        with pytest.raises(ilw.IlwError, match="device"):
            call()


def test_routing_arguments_past_32_bits_are_refused():
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    x = on_gpu((4, 64), torch.float32)
    with pytest.raises(TypeError):
        ilw.moe_route(x, 2, score="sigmoid", scale="much")
    with pytest.raises(OverflowError):
        ilw.moe_route(x, 2, score="sigmoid", groups=1 << 70)


def test_experts_refuse_unknown_arguments_at_once():
    pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    for experts in (ilw.MxExperts, ilw.I8Experts):
        with pytest.raises(TypeError, match="renormalise"):
            experts(None, None, 2, renormalise=False)
        with pytest.raises(TypeError):
            experts(None, None, 2, "silu_gate", None, None, True, "sigmoid")
