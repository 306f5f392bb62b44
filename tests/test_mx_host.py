"""Argument checks of the microscaled 4-bit and mixture-of-experts entry points: validate-only mode, so no kernel runs
and the addresses are never used."""
import ctypes

import pytest

V = ctypes.c_void_p(0x100000)


@pytest.fixture
def L():
    from paper_2607_24981_gb300 import build

    build.build()
    import paper_2607_24981_gb300 as ilw

    lib = ilw.lib()
    assert lib.ilwdetr_validate_only(1) == 0
    yield lib
    lib.ilwdetr_validate_only(0)


def refused(L, rc, code, text):
    assert rc == code and text in L.ilwdetr_last_error(), (rc, L.ilwdetr_last_error())


def test_quantize_checks(L):
    def q(X=V, form=232, ldx=100, x_rows=8, gather=None, rows=8, K=100, codes=V, ldc=64, scales=V, lds=16):
        return L.ilwdetr_mx_quantize(X, form, ldx, x_rows, gather, rows, K, codes, ldc, scales, lds, None)

    assert q() == 0 and q(form=8) == 0 and q(form=216) == 0 and q(form=217, gather=V, rows=50) == 0
    assert q(rows=0, X=None, codes=None, scales=None) == 0
    assert q(X=None, x_rows=0, gather=V) == 0  # every index is then outside: rows of zeros
    refused(L, q(form=16), -1, b"x_form")
    refused(L, q(K=0), -1, b"sizes")
    refused(L, q(ldx=99), -1, b"sizes")
    refused(L, q(rows=9), -1, b"sizes")  # more rows than X has, without a gather
    refused(L, q(X=None), -1, b"NULL")
    refused(L, q(X=ctypes.c_void_p(0x100002)), -1, b"misaligned")
    refused(L, q(codes=ctypes.c_void_p(0x100008)), -1, b"codes")
    refused(L, q(ldc=48), -1, b"codes")
    refused(L, q(ldc=72), -1, b"codes")
    refused(L, q(lds=8), -1, b"scales")
    refused(L, q(scales=None), -1, b"scales")


def test_dequantize_checks(L):
    def d(codes=V, ldc=64, scales=V, lds=16, rows=8, K=100, Y=V, form=217, ldy=100):
        return L.ilwdetr_mx_dequantize(codes, ldc, scales, lds, rows, K, Y, form, ldy, None)

    assert d() == 0 and d(rows=0, codes=None, scales=None, Y=None) == 0
    refused(L, d(form=8), -1, b"y_form")
    refused(L, d(ldy=99), -1, b"sizes")
    refused(L, d(Y=ctypes.c_void_p(0x100001)), -1, b"misaligned")
    refused(L, d(lds=0), -1, b"scales")
    refused(L, d(rows=-1), -1, b"sizes")


def test_gemm_checks(L):
    from paper_2607_24981_gb300 import mx

    fields = dict(a_codes=0x100000, a_ldc=128, a_scales=0x200000, a_lds=16, w_codes=0x300000, w_ldc=128, w_codes_stride=128 * 64,
                  w_scales=0x400000, w_lds=16, w_scales_stride=16 * 64, bias=0, offsets=0, M=300, N=64, K=256, experts=1, act=0, y_form=217,
                  Y=0x500000, ldy=64)

    def g(**over):
        return L.ilwdetr_mx_gemm(mx.gemm_struct(*{**fields, **over}.values()), None)

    assert g() == 0 and g(M=0, Y=0, a_codes=0) == 0 and g(N=0) == 0
    assert g(offsets=0x600000, experts=5, bias=0x700000) == 0
    assert g(act=2, ldy=32) == 0  # a gated result has half the columns
    refused(L, L.ilwdetr_mx_gemm(bytes(200), None), -1, b"struct_size")
    refused(L, L.ilwdetr_mx_gemm(None, None), -1, b"struct_size")
    refused(L, g(act=3), -1, b"act")
    refused(L, g(y_form=8), -1, b"y_form")
    refused(L, g(K=0), -1, b"sizes")
    refused(L, g(experts=2), -1, b"sizes")  # several experts need offsets
    refused(L, g(act=2, N=63), -1, b"even")
    refused(L, g(offsets=0x600000, experts=1025), -2, b"experts")
    refused(L, g(K=(1 << 24) + 1), -2, b"2^24")
    refused(L, g(M=(1 << 31) - 2048, N=1 << 20, ldy=1 << 20), -2, b"too large")
    refused(L, g(a_codes=0x100008), -1, b"a_codes")
    refused(L, g(a_ldc=112), -1, b"a_codes")
    refused(L, g(w_scales=0), -1, b"w_scales")
    refused(L, g(w_lds=24), -1, b"w_scales")
    refused(L, g(offsets=0x600000, experts=5, w_codes_stride=0), -1, b"strides")
    refused(L, g(offsets=0x600000, experts=5, w_scales_stride=1032), -1, b"strides")
    refused(L, g(offsets=0x600002, experts=5), -1, b"misaligned")
    refused(L, g(ldy=63), -1, b"Y")
    refused(L, g(Y=0x500001), -1, b"Y")


def test_route_and_combine_check(L):
    def r(logits=V, form=217, ld=64, T=5000, E=64, k=4, offsets=V, slot=V, ws=V, size=1 << 20):
        return L.ilwdetr_moe_route(logits, form, ld, T, E, k, 1, V, V, offsets, V, slot, ws, size, None)

    assert r() == 0 and r(T=0, logits=None, slot=None) == 0
    assert r(T=16, ws=None, size=0) == 0 and L.ilwdetr_moe_route_workspace_bytes(16, 64) == 0  # one CTA needs none
    refused(L, r(form=8), -1, b"form")
    refused(L, r(k=0), -1, b"sizes")
    refused(L, r(k=65), -1, b"sizes")
    refused(L, r(ld=63), -1, b"sizes")
    refused(L, r(E=513, ld=513), -2, b"512")
    refused(L, r(k=17), -2, b"16")
    refused(L, r(slot=None), -1, b"NULL")
    refused(L, r(offsets=None), -1, b"offsets")
    refused(L, r(logits=ctypes.c_void_p(0x100001)), -1, b"misaligned")
    refused(L, r(size=16), -1, b"workspace")

    def c(Y=V, form=232, ldy=32, rows=20, slot=V, T=10, k=2, N=32, res=None, ldr=0, out=V, ldo=32):
        return L.ilwdetr_moe_combine(Y, form, ldy, rows, slot, V, T, k, N, res, ldr, out, ldo, None)

    assert c() == 0 and c(res=V, ldr=32) == 0 and c(T=0, Y=None, slot=None, out=None) == 0 and c(Y=None, rows=0) == 0
    refused(L, c(form=8), -1, b"form")
    refused(L, c(k=0), -1, b"sizes")
    refused(L, c(ldy=31), -1, b"sizes")
    refused(L, c(res=V, ldr=31), -1, b"sizes")
    refused(L, c(slot=None), -1, b"NULL")
    refused(L, c(out=ctypes.c_void_p(0x100002)), -1, b"misaligned")


def test_binding_refuses_what_it_cannot_pass_on():
    """Checks of the binding itself, on CPU tensors: none reaches the library."""
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    x = torch.zeros(4, 64)
    m = ilw.MxTensor(torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 16, dtype=torch.uint8), 64)
    for call in (lambda: ilw.mx_quantize(x), lambda: ilw.mx_dequantize(m), lambda: ilw.mx_linear(m, m), lambda: ilw.moe_route(x, 2),
                 lambda: ilw.moe_combine(x, torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, 2))):
        with pytest.raises(ilw.IlwError, match="GPU|CUDA"):
            call()
    with pytest.raises(ilw.IlwError, match="2 dimensions|dimensions, not 2"):
        ilw.mx_quantize(torch.zeros(2, 2, 2))
    with pytest.raises(ilw.IlwError, match="MXFP4"):
        ilw.mx_linear(m._replace(k=65), m)
    with pytest.raises(ilw.IlwError, match="GPU"):
        ilw.mx_grouped_linear(m, m, torch.zeros(5, dtype=torch.int32))


def test_binding_fails_loudly_without_its_library(monkeypatch):
    """With _mxbind.so absent a call raises instead of computing anything elsewhere."""
    torch = pytest.importorskip("torch")
    from paper_2607_24981_gb300 import IlwError, mx

    monkeypatch.setattr(mx, "_bound", None)
    monkeypatch.setattr(mx, "BIND_PATH", mx.BIND_PATH + ".absent")
    with pytest.raises(IlwError, match="missing"):
        mx.moe_route(torch.zeros(2, 4), 1)


def on_gpu(size, dtype, device="cuda:0", strides=None):
    """A tensor on a GPU with nothing behind it: the binding's checks of shapes and devices come before any launch or copy."""
    torch = pytest.importorskip("torch")

    class Nowhere(torch.Tensor):
        __torch_function__ = torch._C._disabled_torch_function_impl

        @classmethod
        def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
            raise AssertionError(f"{func} called")

    return torch.Tensor._make_wrapper_subclass(Nowhere, size, dtype=dtype, device=device, strides=strides)


@pytest.mark.parametrize("R,K,width,stride", [(1, 96, 3, 3), (1, 600, 19, 32), (4, 96, 3, 16), (4, 520, 17, 32)])
def test_quantize_refuses_scales_without_room_for_their_padding(R, K, width, stride):
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    codes = on_gpu((R, -(-K // 32) * 16), torch.uint8)
    out = ilw.MxTensor(codes, on_gpu((R, width), torch.uint8, strides=(stride, 1)), K)
    with pytest.raises(ilw.IlwError, match="scales"):
        ilw.mx_quantize(on_gpu((R, K), torch.float32), out=out)


def test_gate_rows_alternate_along_their_axis():
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    for shape, dim, at in (((5,), None, 0), ((5, 7), None, 0), ((3, 5, 7), None, 1), ((3, 5), 1, 1), ((3, 5), -1, 1), ((1, 5), 1, 1), ((3, 5, 7), -2, 1)):
        gate, up = torch.rand(shape), torch.rand(shape)
        got = ilw.gate_rows(gate, up) if dim is None else ilw.gate_rows(gate, up, dim=dim)
        assert got.shape == torch.Size(2 * n if i == at else n for i, n in enumerate(shape))
        for r in range(5):
            assert torch.equal(got.select(at, 2 * r), gate.select(at, r)) and torch.equal(got.select(at, 2 * r + 1), up.select(at, r))


def test_biases_and_weights_of_another_shape_are_refused():
    """As many values in rows of another length would be taken in the wrong order."""
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    E, N, K = 3, 8, 64
    mx = lambda *rows: ilw.MxTensor(on_gpu((*rows, 32), torch.uint8), on_gpu((*rows, 16), torch.uint8), K)  # noqa: E731
    a, w, off = mx(5), mx(E, N), on_gpu((E + 1,), torch.int32)
    for shape in ((N, E), (2 * E, N // 2), (E * N, 1), (E, N + 1), (E + 1, N)):
        with pytest.raises(ilw.IlwError, match="bias"):
            ilw.mx_grouped_linear(a, w, off, bias=on_gpu(shape, torch.float32), act="silu_gate")
    for shape in ((2, N // 2), (N + 1,), (N, 1)):
        with pytest.raises(ilw.IlwError, match="bias"):
            ilw.mx_linear(a, mx(N), bias=on_gpu(shape, torch.float32))
    y, slot = on_gpu((10, 16), torch.float32), on_gpu((5, 2), torch.int32)
    for shape in ((2, 5), (5, 3), (10, 1)):
        with pytest.raises(ilw.IlwError, match="weight"):
            ilw.moe_combine(y, slot, on_gpu(shape, torch.float32))


def test_tensors_of_more_than_one_gpu_are_refused():
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    def mx(rows, at="cuda:0", scales_at=None):
        return ilw.MxTensor(on_gpu((*rows, 32), torch.uint8, at), on_gpu((*rows, 16), torch.uint8, scales_at or at), 64)

    def t(*size, dtype=torch.float32, at="cuda:0"):
        return on_gpu(size, dtype, at)

    far = "cuda:1"
    i32 = torch.int32
    for call in (lambda: ilw.mx_quantize(t(4, 64), gather=t(4, dtype=i32, at=far)), lambda: ilw.mx_quantize(t(4, 64), out=mx((4,), far)),
                 lambda: ilw.mx_quantize(t(4, 64), out=mx((4,), "cuda:0", far)), lambda: ilw.mx_dequantize(mx((4,)), out=t(4, 64, at=far)),
                 lambda: ilw.mx_linear(mx((4,)), mx((8,), far)), lambda: ilw.mx_linear(mx((4,)), mx((8,), "cuda:0", far)),
                 lambda: ilw.mx_linear(mx((4,)), mx((8,)), bias=t(8, at=far)), lambda: ilw.mx_linear(mx((4,)), mx((8,)), out=t(4, 8, at=far)),
                 lambda: ilw.mx_grouped_linear(mx((4,)), mx((2, 8)), t(3, dtype=i32, at=far)),
                 lambda: ilw.moe_combine(t(8, 16), t(4, 2, dtype=i32, at=far), t(4, 2)), lambda: ilw.moe_combine(t(8, 16), t(4, 2, dtype=i32), t(4, 2, at=far)),
                 lambda: ilw.moe_combine(t(8, 16), t(4, 2, dtype=i32), t(4, 2), residual=t(4, 16, at=far)),
                 lambda: ilw.moe_combine(t(8, 16), t(4, 2, dtype=i32), t(4, 2), out=t(4, 16, at=far))):
        with pytest.raises(ilw.IlwError, match="device"):
            call()


@pytest.mark.parametrize("k", [0, -1, -(1 << 40), 2**31, 2**32 + 64])
def test_an_mxfp4_tensor_of_a_k_outside_32_bits_is_refused(k):
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    nb = max(k + 31, 0) // 32
    m = ilw.MxTensor(on_gpu((2, 16 * nb), torch.uint8), on_gpu((2, -(-nb // 16) * 16), torch.uint8), k)
    for call in (lambda: ilw.mx_dequantize(m), lambda: ilw.mx_dequantize(m, out=on_gpu((2, max(k, 0)), torch.float16)), lambda: ilw.mx_linear(m, m)):
        with pytest.raises(ilw.IlwError, match="k="):
            call()


def test_route_passes_on_an_argument_without_a_truth_value():
    torch = pytest.importorskip("torch")
    import paper_2607_24981_gb300 as ilw

    class Neither:
        def __bool__(self):
            raise ArithmeticError("neither")

    with pytest.raises(ArithmeticError, match="neither"):
        ilw.moe_route(on_gpu((4, 8), torch.float32), 2, renormalize=Neither())


def test_the_library_is_built_where_there_is_no_torch(L, monkeypatch):
    """The C-ABI needs none; only the binding of torch tensors does, and is then left out."""
    import sys

    from paper_2607_24981_gb300 import build

    monkeypatch.setitem(sys.modules, "torch", None)  # (an import of it raises ImportError)
    stale = build._stale
    monkeypatch.setattr(build, "_stale", lambda out, deps: out == build.BIND or stale(out, deps))
    at = build.os.path.getmtime(build.BIND)
    assert build.build() == build.LIB and build.os.path.getmtime(build.BIND) == at


def test_a_binding_that_does_not_build_leaves_the_library_built(L, monkeypatch, tmp_path):
    from paper_2607_24981_gb300 import build

    def no_headers(verbose=False):
        raise RuntimeError("no Python.h")

    monkeypatch.setattr(build, "build_binding", no_headers)
    monkeypatch.setattr(build, "BIND", str(tmp_path / "absent.so"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    with pytest.raises(RuntimeError, match="Python.h"):
        build.build()
    assert build.os.path.exists(build.LIB)


def test_a_binding_of_another_python_or_torch_is_built_again(L, monkeypatch):
    from paper_2607_24981_gb300 import build

    built = []
    monkeypatch.setattr(build, "build_binding", lambda verbose=False: built.append(1))
    build.build()
    assert not built
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(torch, "__version__", "0.0")
    build.build()
    assert built


def test_a_binding_that_does_not_load_is_refused(L, monkeypatch):
    import sys

    import paper_2607_24981_gb300 as ilw
    from paper_2607_24981_gb300 import IlwError, mx

    torch = pytest.importorskip("torch")
    monkeypatch.setattr(mx, "_bound", None)
    monkeypatch.setitem(sys.modules, "paper_2607_24981_gb300._mxbind", None)
    monkeypatch.delattr(ilw, "_mxbind", raising=False)
    with pytest.raises(IlwError, match="does not load"):
        mx.moe_route(torch.zeros(2, 4), 1)


def form_of(L, M, N, K, counts=None, act="none", y_form=217, sms=152):
    """(form, CTAs that share a tile's K, tokens a tile) of a product with contiguous operands; `counts`: experts."""
    from paper_2607_24981_gb300 import mx

    nb = -(-K // 32)
    lds, wide = -(-nb // 16) * 16, N // 2 if act == "silu_gate" else N
    got = (ctypes.c_int32 * 3)()
    rc = L.ilwdetr_debug_mx_form(mx.gemm_struct(1 << 20, 16 * nb, 1 << 20, lds, 1 << 20, 16 * nb, N * 16 * nb, 1 << 20, lds, N * lds, 0, 1 << 20 if counts else 0,
                                                M, N, K, counts or 1, mx.ACTS[act], y_form, 1 << 20, wide), sms, got)
    assert rc == 0, L.ilwdetr_last_error()
    return tuple(got)


def test_forms_of_products(L):
    assert form_of(L, 1, 4096, 4096) == (1, 4, 16)
    assert form_of(L, 8192, 8192, 8192) == (2, 1, 224)
    assert form_of(L, 32, 4096, 2048, counts=64, act="silu_gate")[0] == 0
    refused(L, L.ilwdetr_debug_mx_form(None, 152, (ctypes.c_int32 * 3)()), -1, b"struct_size")
    assert L.ilwdetr_debug_mx_form(None, 152, None) == -1


@pytest.mark.parametrize("sms", [132, 148, 152, 160])
def test_forms_keep_to_what_the_kernel_takes(L, sms):
    """Over sizes of all kinds: tiles in steps that the MMA takes, clusters no larger than K has stages and all of them resident at once."""
    import random

    rng = random.Random(sms)
    seen = set()
    for _ in range(4000):
        size = lambda top: int(round(2 ** rng.uniform(0, top)))  # noqa: E731
        M, N, K, E = size(15), 2 * size(13), size(14), rng.choice([None, None, size(10)])
        act = rng.choice(["none", "gelu", "silu_gate"])
        form, splits, tokens = form_of(L, M, N, K, E, act, rng.choice([217, 232]), sms)
        seen.add((form, splits))
        assert 16 <= tokens <= 224 and tokens % (32 if form == 2 else 16) == 0
        tiles = min(M, M // tokens + E) if E else -(-M // tokens)
        if form == 1:
            assert splits in (2, 4, 8) and splits <= -(-K // 512) and splits * tiles * -(-N // 128) <= sms
        else:
            assert splits == 1 and (form == 0 or (N > 128 and K > 1024))
    assert seen == {(0, 1), (1, 2), (1, 4), (1, 8), (2, 1)}
