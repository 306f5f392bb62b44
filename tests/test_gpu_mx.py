"""Microscaled 4-bit and mixture-of-experts operators on the GPU against plain restatements in 64 bits.

Quantisation, its inverse, expert choice and order are exact.  Products: every code product and block scale is exact and
sums are fp32, so whatever the order and even if each addition truncates, |error| <= (K + 8) 2^-23 sum_k |a_k w_k| before
the activation; the activations here have a slope of at most 1.13 (GELU) and take at most 8 further roundings, and the
output is rounded once to its type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

EPS = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}  # half an ulp, relative
LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


@pytest.fixture(scope="module")
def ilw():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2607_24981_gb300 as m
    from paper_2607_24981_gb300 import build

    build.build()
    m.lib()
    return m


# ---------------------------------------------------------------------------- restatements
def ref_quantize(x):
    """Codes [R, blocks * 32] and scale bytes [R, blocks] of float64 x [R, K]."""
    R, K = x.shape
    nb = -(-K // 32)
    v = np.zeros((R, nb * 32))
    v[:, :K] = x
    neg = np.zeros(v.shape, bool)
    neg[:, :K] = np.signbit(x)
    v = v.reshape(R, nb, 32)
    amax = np.abs(v).max(2)
    byte = np.full(amax.shape, 255)
    fine = np.isfinite(amax)
    exponent = np.frexp(np.where(fine, amax, 1))[1] - 1
    byte[fine] = (np.clip(exponent - 2, -127, 127) + 127)[fine]
    byte[amax == 0] = 0
    with np.errstate(invalid="ignore"):
        y = np.abs(v) / np.ldexp(1.0, byte - 127)[:, :, None]
    d = np.abs(np.minimum(np.where(np.isfinite(y), y, 0), 6.0)[..., None] - LEVELS)
    d[..., 1::2] += 1e-9  # ties go to the even code (no distance of these inputs is within 1e-9 of another but a tie)
    code = d.argmin(-1).reshape(R, -1) + 8 * neg
    code[np.repeat(byte == 255, 32, axis=1)] = 0
    return code, byte


def ref_values(codes, scales, k):
    """Float64 values of uint8 codes [.., R, 16 nb] and scales (numpy)."""
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = LEVELS[nib & 7] * np.where(nib & 8, -1.0, 1.0)
    s = np.ldexp(1.0, scales.astype(np.int64) - 127)
    s[scales == 255] = np.nan
    return (v * np.repeat(s, 32, axis=-1)[..., : v.shape[-1]])[..., :k]


def ref_act(z, act):
    from math import erf

    if act == "gelu":
        return 0.5 * z * (1 + np.vectorize(erf)(z / np.sqrt(2)))
    if act == "silu_gate":
        g, u = z[:, 0::2], z[:, 1::2]
        return g / (1 + np.exp(-g)) * u
    return z


def host(m):
    return m.codes.cpu().numpy(), m.scales.cpu().numpy()


def packed(ilw, x):
    """x float64 numpy [.., R, K] as an MxTensor made on the host."""
    R, K = x.shape[-2:]
    code, byte = ref_quantize(x.reshape(-1, K))
    nb = byte.shape[1]
    codes = (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)
    scales = np.full((codes.shape[0], -(-nb // 16) * 16), 255, np.uint8)  # bytes past the row's blocks are not read
    scales[:, :nb] = byte
    lead = x.shape[:-1]
    return ilw.MxTensor(torch.from_numpy(codes.reshape(*lead, -1)).cuda(), torch.from_numpy(scales.reshape(*lead, -1)).cuda(), K)


def check_product(got, a, w, bias, act, dtype):
    """got [M, n] against the 64-bit product of values a [M, K], w [N, K]; the bound of the module's docstring."""
    z, mass = a @ w.T, np.abs(a) @ np.abs(w).T
    if bias is not None:
        z, mass = z + bias, mass + np.abs(bias)
    tol = (a.shape[1] + 8) * 2.0**-23 * mass
    want = ref_act(z, act)
    if act == "silu_gate":
        g, u = z[:, 0::2], z[:, 1::2]
        s = 1 / (1 + np.exp(-g))
        tol = 1.1 * tol[:, 0::2] * (np.abs(u) + tol[:, 1::2]) + np.abs(g * s) * tol[:, 1::2] + 8 * 2.0**-24 * np.abs(want)
    elif act == "gelu":
        tol = 1.13 * tol + 8 * 2.0**-24 * np.abs(z)
    tol = tol + EPS[dtype] * (np.abs(want) + tol) + (2.0**-25 if dtype == torch.float16 else 0.0)  # (a subnormal's half ulp)
    err = np.abs(got.double().cpu().numpy() - want)
    assert got.dtype == dtype and got.shape == want.shape
    assert (err <= tol).all(), f"{(err > tol).sum()} of {err.size} outside, worst {np.max(err / tol):.3g} times the bound"


def values(rng, R, K):
    """Rows of very different sizes, a few of them zero."""
    x = rng.standard_normal((R, K)) * np.exp2(rng.integers(-6, 7, (R, 1)))
    x[rng.random(R) < 0.1] = 0
    return x


# ---------------------------------------------------------------------------- quantisation
FORMS = [torch.float32, torch.float16, torch.bfloat16, torch.int8]


@pytest.mark.parametrize("dtype", FORMS)
@pytest.mark.parametrize("R,K", [(1, 1), (3, 31), (2, 32), (5, 33), (4, 264), (7, 257), (2, 2051), (130, 520)])
def test_quantize_matches_64_bits(ilw, dtype, R, K):
    rng = np.random.default_rng(R * 1000 + K)
    x = torch.from_numpy(values(rng, R, K) * 4).clamp(-127, 127)
    x = (x.round() if dtype == torch.int8 else x).to(dtype).cuda()
    m = ilw.mx_quantize(x)
    code, byte = ref_quantize(x.double().cpu().numpy())
    codes, scales = host(m)
    assert (codes == (code[:, 0::2] | code[:, 1::2] << 4)).all()
    assert (scales[:, : byte.shape[1]] == byte).all() and (scales[:, byte.shape[1]:] == 0).all()
    for out in (torch.float32, torch.float16, torch.bfloat16):
        want = torch.from_numpy(ref_values(codes, scales, K)).to(out).cuda()
        assert torch.equal(ilw.mx_dequantize(m, out), want)


def test_quantize_special_values(ilw):
    """Ties, powers of two, subnormals, the largest values, signed zeros, infinities and NaN."""
    rows = [np.zeros(64), np.full(64, -0.0), np.tile(LEVELS, 8), np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0], 8),
            -np.tile([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], 8) * 2.0**-40, np.full(64, 3.4028234e38), np.full(64, 2.0**-149),
            np.exp2(np.arange(64) - 140.0), np.exp2(-np.arange(64.0)), np.r_[np.inf, np.ones(63)], np.r_[np.ones(40), np.nan, np.ones(23)],
            np.r_[np.full(32, -np.inf), np.ones(32)], np.full(64, 2.0**-126), np.full(64, 1.5 * 2.0**-127)]
    x = torch.from_numpy(np.stack(rows)).float()
    m = ilw.mx_quantize(x.cuda())
    code, byte = ref_quantize(x.double().numpy())
    codes, scales = host(m)
    assert (scales[:, :2] == byte).all()
    assert (codes == (code[:, 0::2] | code[:, 1::2] << 4)).all()
    back = ilw.mx_dequantize(m).cpu().numpy()
    assert np.isnan(back[9, :32]).all() and np.isfinite(back[9, 32:]).all() and np.isnan(back[10, 32:]).all()
    assert np.array_equal(back, ref_values(codes, scales, 64).astype(np.float32), equal_nan=True)


def test_quantize_gathers_rows(ilw):
    rng = np.random.default_rng(3)
    x = torch.from_numpy(values(rng, 50, 300)).float().cuda()
    at = torch.from_numpy(rng.integers(-1, 50, 77).astype(np.int32)).cuda()
    m, whole = ilw.mx_quantize(x, gather=at), ilw.mx_quantize(x)
    rows = at.long()
    assert torch.equal(m.codes, torch.where(rows[:, None] < 0, 0, whole.codes[rows]))
    assert torch.equal(m.scales, torch.where(rows[:, None] < 0, 0, whole.scales[rows]))
    ilw.device_status()
    bad = torch.tensor([0, 50, -2, 49], dtype=torch.int32, device="cuda")
    m = ilw.mx_quantize(x, gather=bad)
    assert (m.codes[1:3] == 0).all() and (m.scales[1:3] == 0).all() and torch.equal(m.codes[3], whole.codes[49])
    with pytest.raises(ilw.IlwError, match="index"):
        ilw.device_status()
    ilw.device_status()


@pytest.mark.parametrize("dtype", FORMS)
def test_quantize_rows_with_strides_and_offsets(ilw, dtype):
    """Rows inside a wider tensor, starting off 16-byte boundaries; results into rows of a wider one, the rest untouched."""
    rng = np.random.default_rng(4)
    wide = torch.from_numpy(np.clip(values(rng, 9, 200), -127, 127)).to(dtype).cuda()
    for lo, hi in ((3, 100), (16, 112), (1, 2)):
        x = wide[:, lo:hi]
        want = ilw.mx_quantize(x.contiguous())
        assert all(torch.equal(p, q) for p, q in zip(ilw.mx_quantize(x)[:2], want[:2]))
        n, s = want.codes.shape[1], want.scales.shape[1]
        codes = torch.full((9, n + 32), 77, dtype=torch.uint8, device="cuda")
        scales = torch.full((9, s + 16), 77, dtype=torch.uint8, device="cuda")
        out = ilw.MxTensor(codes[:, 16: 16 + n], scales[:, :s], hi - lo)
        ilw.mx_quantize(x, out=out)
        assert torch.equal(out.codes, want.codes) and torch.equal(out.scales, want.scales)
        assert (codes[:, :16] == 77).all() and (codes[:, 16 + n:] == 77).all() and (scales[:, s:] == 77).all()


@pytest.mark.parametrize("R,K,width,stride", [(1, 96, 3, 3), (1, 600, 19, 19), (4, 96, 3, 16), (4, 96, 15, 32), (2, 544, 31, 32)])
def test_quantize_keeps_to_the_scales_it_is_given(ilw, R, K, width, stride):
    """Scales of out narrower than the 16 bytes that a row is filled up to: refused, and nothing around them is written."""
    guard = torch.full((16 + (R - 1) * stride + width + 64,), 77, dtype=torch.uint8, device="cuda")
    codes = torch.full((R, K // 32 * 16 + 16), 77, dtype=torch.uint8, device="cuda")[:, : -(-K // 32) * 16]
    out = ilw.MxTensor(codes, guard[16:].as_strided((R, width), (stride, 1)), K)
    x = torch.ones((R, K), device="cuda")
    with pytest.raises(ilw.IlwError, match="scales"):
        ilw.mx_quantize(x, out=out)
    assert (guard == 77).all() and (codes == 77).all()
    padded = -(-width // 16) * 16
    out = out._replace(scales=guard[16:].as_strided((R, padded), (max(stride, padded), 1))) if R == 1 else out._replace(scales=torch.zeros((R, padded), dtype=torch.uint8, device="cuda"))
    ilw.mx_quantize(x, out=out)
    want = ilw.mx_quantize(x)
    assert torch.equal(out.codes, want.codes) and torch.equal(out.scales, want.scales)
    assert (guard[:16] == 77).all() and (guard[16 + padded:] == 77).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_dequantize_every_code_and_scale(ilw, dtype):
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scales = np.tile(np.arange(256, dtype=np.uint8)[:, None], (1, 16))
    m = ilw.MxTensor(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), 512)
    want = torch.from_numpy(ref_values(codes, scales, 512)).float().to(dtype)
    got = ilw.mx_dequantize(m, dtype).cpu()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~got.isnan()], want[~want.isnan()])
    out = torch.full((256, 520), 7.0, dtype=dtype, device="cuda")
    for lo, k in ((1, 511), (8, 512), (0, 1)):  # rows off 16-byte boundaries, and odd widths
        part = ilw.mx_dequantize(ilw.MxTensor(m.codes, m.scales, k), out=out[:, lo: lo + k]).cpu()
        assert torch.equal(part.nan_to_num(3.0), want[:, :k].nan_to_num(3.0))
        assert (out[:, :lo] == 7).all() and (out[:, lo + k:] == 7).all()
        out.fill_(7)


def test_quantize_and_back_of_more_than_2_32_threads(ilw):
    """Short rows off 16-byte boundaries, a warp each: 2^27 of them are 2^32 threads."""
    R = 2**27 + 300
    x = (torch.arange(R, dtype=torch.int32, device="cuda") % 6 + 1).to(torch.int8)[:, None]  # 1 to 6, as 4 or 6 times a power of two; 5: as 4 or 6
    m = ilw.mx_empty(R, 1)
    m.codes.fill_(255), m.scales.fill_(255)
    ilw.mx_quantize(x, out=m)
    few = ilw.mx_quantize(x[:6].clone())
    for got, want in ((m.codes, few.codes), (m.scales, few.scales)):
        assert bool((got[: R // 6 * 6].view(-1, 6, 16) == want).all()) and torch.equal(got[R // 6 * 6:], want[: R % 6])
    out = torch.full((R, 1), -1.0, dtype=torch.float16, device="cuda")
    ilw.mx_dequantize(m, out=out)
    want = ilw.mx_dequantize(few, torch.float16)
    assert bool((out[: R // 6 * 6].view(-1, 6) == want[:, 0]).all()) and torch.equal(out[R // 6 * 6:], want[: R % 6])


# ---------------------------------------------------------------------------- products
@pytest.mark.parametrize("act,bias", [("none", False), ("none", True), ("gelu", True), ("silu_gate", False), ("silu_gate", True)])
@pytest.mark.parametrize("M,N,K", [(1, 2, 1), (1, 128, 4096), (3, 130, 512), (16, 300, 33), (17, 128, 250), (33, 1000, 2048),
                                   (224, 256, 768), (225, 126, 1100), (700, 514, 96)])
def test_linear_matches_64_bits(ilw, M, N, K, act, bias):
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    A, W = packed(ilw, values(rng, M, K)), packed(ilw, rng.standard_normal((N, K)) / np.sqrt(K))
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    a, w = ref_values(*host(A), K), ref_values(*host(W), K)
    for dtype in (torch.float32, torch.bfloat16):
        got = ilw.mx_linear(A, W, None if b is None else torch.from_numpy(b).cuda(), act=act, out_dtype=dtype)
        check_product(got, a, w, b, act, dtype)
    ilw.device_status()


@pytest.mark.parametrize("splits,K", [(2, 1024), (4, 2048 + 32), (8, 8192 + 300)])
def test_linear_of_few_tiles(ilw, splits, K):
    """One to three tiles, whose K is shared by several CTAs: the same bound, and the same bits on every run."""
    rng = np.random.default_rng(K)
    for M, N in ((1, 128), (5, 300), (200, 64)):
        A, W = packed(ilw, values(rng, M, K)), packed(ilw, rng.standard_normal((N, K)) / np.sqrt(K))
        a, w = ref_values(*host(A), K), ref_values(*host(W), K)
        got = ilw.mx_linear(A, W, out_dtype=torch.float32)
        check_product(got, a, w, None, "none", torch.float32)
        assert all(torch.equal(got, ilw.mx_linear(A, W, out_dtype=torch.float32)) for _ in range(5))


@pytest.mark.parametrize("act,K", [("none", 32), ("none", 1300), ("gelu", 2100), ("silu_gate", 4096)])
def test_linear_of_many_tiles(ilw, act, K):
    """As many tiles as two SMs share each (256 outputs, up to 224 tokens), over one to eight stages of scales; the same bits again."""
    rng = np.random.default_rng(K)
    M, N = 3001, 1700
    A, W = packed(ilw, values(rng, M, K)), packed(ilw, rng.standard_normal((N, K)) / np.sqrt(K))
    a, w = ref_values(*host(A), K), ref_values(*host(W), K)
    for dtype in (torch.float32, torch.bfloat16):
        got = ilw.mx_linear(A, W, act=act, out_dtype=dtype)
        check_product(got, a, w, None, act, dtype)
        assert all(torch.equal(got, ilw.mx_linear(A, W, act=act, out_dtype=dtype)) for _ in range(3))
    ilw.device_status()


@pytest.mark.parametrize("K,act", [(200, "none"), (1600, "silu_gate")])
def test_grouped_of_many_tiles(ilw, K, act):
    """Long ragged groups, whose tiles two SMs share."""
    rng = np.random.default_rng(K)
    counts, N = [700, 0, 1, 333, 1024, 225, 95], 2304
    off = np.r_[0, np.cumsum(counts)]
    A, W = packed(ilw, values(rng, int(off[-1]), K)), packed(ilw, rng.standard_normal((len(counts), N, K)) / np.sqrt(K))
    a, w = ref_values(*host(A), K), ref_values(*host(W), K)
    for dtype in (torch.float32, torch.bfloat16):
        got = ilw.mx_grouped_linear(A, W, torch.from_numpy(off.astype(np.int32)).cuda(), act=act, out_dtype=dtype)
        for e in range(len(counts)):
            if counts[e]:
                check_product(got[off[e]: off[e + 1]], a[off[e]: off[e + 1]], w[e], None, act, dtype)
    ilw.device_status()


@pytest.mark.parametrize("act,dtype", [("none", torch.float32), ("gelu", torch.bfloat16), ("silu_gate", torch.float16)])
@pytest.mark.parametrize("M,N,K", [(4, 5000, 8200), (9, 1300, 4200), (1, 130, 4128), (224, 900, 9000), (506, 18, 3178), (3, 300, 3500)])
def test_linear_of_a_long_sum(ilw, M, N, K, act, dtype):
    """Few tiles and a long K, which two, four or eight CTAs share: the same bound, and the same bits on every run."""
    rng = np.random.default_rng(M + N + K)
    A, W = packed(ilw, values(rng, M, K)), packed(ilw, rng.standard_normal((N, K)) / np.sqrt(K))
    b = rng.standard_normal(N).astype(np.float32)
    got = ilw.mx_linear(A, W, torch.from_numpy(b).cuda(), act=act, out_dtype=dtype)
    check_product(got, ref_values(*host(A), K), ref_values(*host(W), K), b, act, dtype)
    assert all(torch.equal(got, ilw.mx_linear(A, W, torch.from_numpy(b).cuda(), act=act, out_dtype=dtype)) for _ in range(3))
    ilw.device_status()


@pytest.mark.parametrize("act,dtype", [("none", torch.float32), ("none", torch.bfloat16), ("gelu", torch.float16), ("silu_gate", torch.bfloat16)])
@pytest.mark.parametrize("M,N,K", [(4001, 1700, 3000), (3000, 2306, 2080)])
def test_linear_of_many_long_tiles(ilw, M, N, K, act, dtype):
    """Tiles that two SMs share, several a pair, with a K that ends inside a block; the same bits again."""
    rng = np.random.default_rng(M + N + K)
    A, W = packed(ilw, values(rng, M, K)), packed(ilw, rng.standard_normal((N, K)) / np.sqrt(K))
    b = rng.standard_normal(N).astype(np.float32)
    got = ilw.mx_linear(A, W, torch.from_numpy(b).cuda(), act=act, out_dtype=dtype)
    check_product(got, ref_values(*host(A), K), ref_values(*host(W), K), b, act, dtype)
    assert all(torch.equal(got, ilw.mx_linear(A, W, torch.from_numpy(b).cuda(), act=act, out_dtype=dtype)) for _ in range(3))
    ilw.device_status()


@pytest.mark.parametrize("counts,N,K", [([700, 0, 1, 333, 1024, 225, 95], 2304, 3000), ([1, 0, 9], 300, 4200), ([0, 2, 130, 0], 140, 8192)],
                         ids=["pairs", "eight a tile", "rows of two tiles"])
def test_grouped_with_a_long_sum(ilw, counts, N, K):
    """Ragged groups in the forms for many tiles and for few."""
    rng = np.random.default_rng(N + K)
    off = np.r_[0, np.cumsum(counts)]
    A, W = packed(ilw, values(rng, int(off[-1]), K)), packed(ilw, rng.standard_normal((len(counts), N, K)) / np.sqrt(K))
    a, w = ref_values(*host(A), K), ref_values(*host(W), K)
    for dtype, act in ((torch.float32, "none"), (torch.bfloat16, "silu_gate")):
        got = ilw.mx_grouped_linear(A, W, torch.from_numpy(off.astype(np.int32)).cuda(), act=act, out_dtype=dtype)
        for e in range(len(counts)):
            if counts[e]:
                check_product(got[off[e]: off[e + 1]], a[off[e]: off[e + 1]], w[e], None, act, dtype)
    ilw.device_status()


def form_of(ilw, M, N, K, experts, act, dtype):
    """What the library takes for a product with contiguous operands on this GPU: "one" CTA a tile, "pair" of SMs, or how many CTAs
    share a tile's K; and the tokens of a tile."""
    import ctypes

    from paper_2607_24981_gb300 import mx

    nb, got = -(-K // 32), (ctypes.c_int32 * 3)()
    lds, wide = -(-nb // 16) * 16, N // 2 if act == "silu_gate" else N
    y_form = {torch.float32: 232, torch.float16: 216, torch.bfloat16: 217}[dtype]
    rc = ilw.lib().ilwdetr_debug_mx_form(mx.gemm_struct(1 << 20, 16 * nb, 1 << 20, lds, 1 << 20, 16 * nb, N * 16 * nb, 1 << 20, lds, N * lds, 0, 1 << 20 if experts else 0,
                                                        M, N, K, experts or 1, mx.ACTS[act], y_form, 1 << 20, wide), 0, got)
    assert rc == 0, ilw.lib().ilwdetr_last_error()
    return ["one", got[1], "pair"][got[0]], got[2]


def made(ilw, seed, R, K, weights=False):
    """Weights, or activations in rows of different sizes, as MXFP4 (by mx_quantize, which has its own tests)."""
    gen = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn((R, K), generator=gen, device="cuda")
    return ilw.mx_quantize(x / K**0.5 if weights else x * torch.exp2(torch.randint(-6, 4, (R, 1), generator=gen, device="cuda").float()))


def check_product_on_gpu(ilw, got, A, W, bias, act):
    """check_product with its 64-bit product on the GPU: got [M, n], MXFP4 A and W, fp32 bias or None."""
    a, w = ilw.mx_dequantize(A).double(), ilw.mx_dequantize(W).double()
    z, mass = a @ w.T, a.abs() @ w.abs().T
    if bias is not None:
        z, mass = z + bias.double(), mass + bias.double().abs()
    tol = (A.k + 8) * 2.0**-23 * mass
    if act == "silu_gate":
        g, u = z[:, 0::2], z[:, 1::2]
        s = torch.sigmoid(g)
        want = g * s * u
        tol = 1.1 * tol[:, 0::2] * (u.abs() + tol[:, 1::2]) + (g * s).abs() * tol[:, 1::2] + 8 * 2.0**-24 * want.abs()
    elif act == "gelu":
        want = 0.5 * z * torch.erfc(-z / 2**0.5)
        tol = 1.13 * tol + 8 * 2.0**-24 * z.abs()
    else:
        want = z
    tol = tol + EPS[got.dtype] * (want.abs() + tol) + (2.0**-25 if got.dtype == torch.float16 else 0.0)
    err = (got.double() - want).abs()
    assert got.shape == want.shape and (err <= tol).all(), f"{int((err > tol).sum())} of {err.numel()} outside, worst {float((err / tol).max()):.3g} times the bound"


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("form,M,N,K,act,bias", [
    ("pair", 1500, 1712, 8200, "none", True), ("pair", 1500, 1712, 8200, "gelu", True), ("pair", 1500, 1712, 8200, "silu_gate", True),
    ("pair", 1500, 1712, 8200, "gelu", False), ("pair", 1570, 1701, 8200, "none", True), ("pair", 1570, 1701, 8200, "gelu", True),
    ("pair", 1570, 1702, 8200, "silu_gate", False),
    (8, 5, 1000, 4096, "gelu", True), (8, 40, 1000, 4200, "silu_gate", True), (8, 1, 257, 8000, "none", True),
    (4, 5, 2600, 4128, "silu_gate", True), (4, 200, 1000, 6200, "gelu", True), (4, 100, 1001, 4200, "none", False),
    (2, 5, 6000, 6200, "gelu", True), (2, 224, 2000, 9000, "silu_gate", True), (2, 224, 1999, 9000, "none", True),
    ("one", 1500, 1712, 1000, "gelu", True), ("one", 1500, 1712, 1000, "silu_gate", True), ("one", 333, 1701, 1000, "none", True)])
def test_every_form_with_every_activation(ilw, form, M, N, K, act, bias, dtype):
    assert form_of(ilw, M, N, K, None, act, dtype)[0] == form
    A, W = made(ilw, 1, M, K), made(ilw, 2, N, K, weights=True)
    b = torch.randn(N, device="cuda", generator=torch.Generator("cuda").manual_seed(3)) if bias else None
    got = ilw.mx_linear(A, W, b, act=act, out_dtype=dtype)
    check_product_on_gpu(ilw, got, A, W, b, act)
    assert all(torch.equal(got, ilw.mx_linear(A, W, b, act=act, out_dtype=dtype)) for _ in range(3))
    ilw.device_status()


@pytest.mark.parametrize("M,tokens", [(65, 96), (100, 128), (130, 160), (165, 192), (200, 224), (250, 224)])
def test_pairs_on_tiles_of_every_width(ilw, M, tokens):
    N, K = 19008, 8200
    assert form_of(ilw, M, N, K, None, "gelu", torch.bfloat16) == ("pair", tokens)
    A, W = made(ilw, 1, M, K), made(ilw, 2, N, K, weights=True)
    b = torch.randn(N, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    check_product_on_gpu(ilw, ilw.mx_linear(A, W, b, act="gelu"), A, W, b, "gelu")
    ilw.device_status()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("form,counts,N,K,act", [
    ("pair", [700, 0, 1, 333, 1024, 225, 95], 2304, 2600, "none"), ("pair", [700, 0, 1, 333, 1024, 225, 95], 2304, 2600, "gelu"),
    ("pair", [700, 0, 1, 333, 1024, 225, 95], 2304, 2600, "silu_gate"), (8, [1, 0, 9], 300, 4200, "gelu"), (4, [0, 2, 130, 0], 140, 8192, "silu_gate"),
    ("one", [700, 0, 1, 333, 1024, 225, 95], 1704, 600, "gelu")])
def test_every_form_by_expert(ilw, form, counts, N, K, act, dtype):
    off, E = np.r_[0, np.cumsum(counts)], len(counts)
    assert form_of(ilw, int(off[-1]), N, K, E, act, dtype)[0] == form
    A, W = made(ilw, 1, int(off[-1]), K), made(ilw, 2, E * N, K, weights=True)
    W = ilw.MxTensor(W.codes.view(E, N, -1), W.scales.view(E, N, -1), K)
    b = torch.randn((E, N), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    got = ilw.mx_grouped_linear(A, W, torch.from_numpy(off.astype(np.int32)).cuda(), b, act=act, out_dtype=dtype)
    for e in range(E):
        if counts[e]:
            s = slice(int(off[e]), int(off[e + 1]))
            check_product_on_gpu(ilw, got[s], ilw.MxTensor(A.codes[s], A.scales[s], K), ilw.MxTensor(W.codes[e], W.scales[e], K), b[e], act)
    ilw.device_status()


@pytest.mark.parametrize("form,M,N,K", [("one", 300, 256, 2048), (8, 4, 256, 8192), (4, 5, 2600, 4128), (2, 5, 6000, 6200), ("pair", 3001, 1700, 4096)])
def test_every_form_gives_up_a_bounded_wait(ilw, form, M, N, K):
    """As test_product_gives_up_a_bounded_wait, with the form that each product takes."""
    assert form_of(ilw, M, N, K, None, "none", torch.bfloat16)[0] == form
    A, W = made(ilw, 1, M, K), made(ilw, 2, N, K, weights=True)
    want = ilw.mx_linear(A, W)
    assert ilw.lib().ilwdetr_debug_gemm_wait(0, 20_000_000) == 0
    try:
        ilw.mx_linear(A, W)
        with pytest.raises(ilw.IlwError, match="wait"):
            ilw.device_status()
    finally:
        assert ilw.lib().ilwdetr_debug_gemm_wait(-1, 0) == 0
    assert torch.equal(ilw.mx_linear(A, W), want)
    ilw.device_status()


def test_linear_rows_with_strides(ilw):
    """Operands inside wider byte arrays, a result inside a wider tensor, fp16."""
    rng = np.random.default_rng(11)
    M, N, K = 70, 90, 200
    A, W = packed(ilw, values(rng, M, K)), packed(ilw, rng.standard_normal((N, K)) / np.sqrt(K))
    want = ilw.mx_linear(A, W, out_dtype=torch.float16)
    check_product(want, ref_values(*host(A), K), ref_values(*host(W), K), None, "none", torch.float16)

    def spread(m):
        c = torch.full((m.codes.shape[0], m.codes.shape[1] + 48), 0x77, dtype=torch.uint8, device="cuda")
        s = torch.full((m.scales.shape[0], 64), 255, dtype=torch.uint8, device="cuda")
        c[:, 32: 32 + m.codes.shape[1]] = m.codes
        s[:, 16: 16 + m.scales.shape[1]] = m.scales
        return ilw.MxTensor(c[:, 32: 32 + m.codes.shape[1]], s[:, 16: 16 + m.scales.shape[1]], m.k)

    out = torch.full((M, N + 9), 5.0, dtype=torch.float16, device="cuda")
    ilw.mx_linear(spread(A), spread(W), out=out[:, 3: 3 + N])
    assert torch.equal(out[:, 3: 3 + N], want) and (out[:, :3] == 5).all() and (out[:, 3 + N:] == 5).all()


def test_linear_scales_and_nan(ilw):
    """Block scales far from one (their product near it), and NaN blocks: only their rows and columns are NaN."""
    rng = np.random.default_rng(12)
    M, N, K = 40, 140, 320
    A, W = packed(ilw, values(rng, M, K)), packed(ilw, rng.standard_normal((N, K)))
    A.scales[:, :10] += 100
    W.scales[:, :10] -= 100
    got = ilw.mx_linear(A, W, out_dtype=torch.float32)
    check_product(got, ref_values(*host(A), K), ref_values(*host(W), K), None, "none", torch.float32)
    A.scales[7, 3], W.scales[133, 9] = 255, 255
    bad = ilw.mx_linear(A, W, out_dtype=torch.float32)
    nan = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    nan[7], nan[:, 133] = True, True
    assert torch.equal(bad.isnan(), nan) and torch.equal(bad[~nan], got[~nan])


def through(ilw, z, act, dtype, split):
    """act(z) as a product gives it: zeros times zeros, with the values as its bias (fp32 z [n], 64 rows; split: their K shared)."""
    n, K = z.numel(), 8192 if split else 32
    zero = lambda rows: ilw.MxTensor(torch.zeros((rows, K // 2), dtype=torch.uint8, device="cuda"), torch.zeros((rows, -(-K // 512) * 16), dtype=torch.uint8, device="cuda"), K)  # noqa: E731
    got = ilw.mx_linear(zero(5), zero(n), bias=z, act=act, out_dtype=dtype)
    assert all(torch.equal(got[0].nan_to_num(3.0), got[i].nan_to_num(3.0)) for i in range(1, 5))
    return got[0]


@pytest.mark.parametrize("split", [False, True])
def test_gelu_in_fp32_is_that_of_fp32(ilw, split):
    """erff is off by 2 ulp at most (2^-23), its argument's rounding adds 2^-24 and that of 1 + erf 2^-24: |z| / 2 times that
    and two roundings of the result.  In norm no more than a quarter above plain fp32 operations."""
    n = 1024 if split else 1 << 18
    for z in (torch.linspace(-12, 12, n, device="cuda"), torch.randn(n, device="cuda", generator=torch.Generator("cuda").manual_seed(1))):
        got = through(ilw, z, "gelu", torch.float32, split).double()
        want = 0.5 * z.double() * torch.erfc(-z.double() / 2**0.5)
        plain = (0.5 * z * (1 + torch.erf(z * 0.5**0.5))).double()
        assert ((got - want).abs() <= 2.0**-23 * (z.double().abs() + want.abs())).all()
        assert (got - want).norm() <= 1.25 * (plain - want).norm()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("split", [False, True])
def test_silu_gates_of_every_size(ilw, split, dtype):
    """fp32: an exponential off by 1 ulp (2^-23), the sum, the quotient and two products by 2^-24 each; bf16 by its rounding and
    some 100 of those ulp.  No gate is flushed to zero before exp(-gate) overflows (below -88.7)."""
    n = 512 if split else 1 << 17
    for lo, hi in ((-8, 8), (-87.3, -8), (8, 100)):
        gate = torch.linspace(lo, hi, n, device="cuda")
        up = torch.randn(n, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
        got = through(ilw, torch.stack([gate, up], 1).flatten(), "silu_gate", dtype, split).double()
        want = gate.double() * torch.sigmoid(gate.double()) * up.double()
        tol = 3 * 2.0**-23 if dtype == torch.float32 else 2.0**-8 + 128 * 2.0**-23
        assert ((got - want).abs() <= tol * want.abs() + 2.0**-133).all()  # (a subnormal's rounding)
    gate = torch.linspace(-200, -87.3, n, device="cuda")  # below -88.7 exp(-gate) is infinity in fp32
    got = through(ilw, torch.stack([gate, torch.full_like(gate, 2.0**100)], 1).flatten(), "silu_gate", dtype, split).double()
    want = gate.double() * torch.sigmoid(gate.double()) * 2.0**100
    close = (got - want).abs() <= 2.0**-7 * want.abs()
    assert close[gate >= -88.7].all() and (close | (got == 0)).all()
    special = torch.tensor([float("inf"), 2.0, float("nan"), 1.0, 1.0, float("nan"), 0.0, float("-inf"), -3.0, float("inf"), -0.0, 1.0, 3e38, 1.0, -3e38, 1.0], device="cuda")
    got = through(ilw, special, "silu_gate", dtype, False)
    assert got[0] == float("inf") and got[1:4].isnan().all() and got[4] == float("-inf") and got[5] == 0
    assert got[6] == torch.tensor(3e38, dtype=dtype) and got[7] == 0


GROUPS = {
    "one row each": [1] * 7, "empty ones": [0, 5, 0, 0, 33, 0], "one takes all": [0, 0, 300, 0], "odd": [17, 226, 1, 449, 15],
    "none": [0, 0, 0], "many": [(7 * i) % 5 for i in range(200)],
}


@pytest.mark.parametrize("counts", GROUPS.values(), ids=GROUPS.keys())
@pytest.mark.parametrize("N,K,act", [(130, 100, "none"), (256, 1536, "silu_gate"), (66, 544, "gelu")])
def test_grouped_matches_64_bits(ilw, counts, N, K, act):
    """Ragged groups between rows of no expert (before the first and after the last), which come out zero."""
    rng = np.random.default_rng(N + K + len(counts))
    E, head, tail = len(counts), 3, 5
    off = head + np.r_[0, np.cumsum(counts)]
    M = int(off[-1]) + tail
    A, W = packed(ilw, values(rng, M, K)), packed(ilw, rng.standard_normal((E, N, K)) / np.sqrt(K))
    b = rng.standard_normal((E, N)).astype(np.float32)
    a, w = ref_values(*host(A), K), ref_values(*host(W), K)
    for dtype in (torch.float32, torch.bfloat16):
        got = ilw.mx_grouped_linear(A, W, torch.from_numpy(off.astype(np.int32)).cuda(), torch.from_numpy(b).cuda(), act=act, out_dtype=dtype)
        assert (got[:head] == 0).all() and (got[off[-1]:] == 0).all()
        for e in range(E):
            if counts[e]:
                check_product(got[off[e]: off[e + 1]], a[off[e]: off[e + 1]], w[e], b[e], act, dtype)
    ilw.device_status()


def test_grouped_of_very_many_experts(ilw):
    """The table of 1024 experts takes shared memory from the widest tiles."""
    rng = np.random.default_rng(21)
    E, N, K = 1024, 64, 100
    counts = 90 + 40 * (np.arange(E) % 2)
    off = np.r_[0, np.cumsum(counts)]
    A, W = packed(ilw, values(rng, int(off[-1]), K)), packed(ilw, rng.standard_normal((E, N, K)) / np.sqrt(K))
    a, w = ref_values(*host(A), K), ref_values(*host(W), K)
    got = ilw.mx_grouped_linear(A, W, torch.from_numpy(off.astype(np.int32)).cuda(), act="gelu", out_dtype=torch.bfloat16)
    for e in range(E):
        check_product(got[off[e]: off[e + 1]], a[off[e]: off[e + 1]], w[e], None, "gelu", torch.bfloat16)
    ilw.device_status()


def test_grouped_survives_bad_offsets(ilw):
    """Offsets out of order and range: no access outside the tensors (rows come out wrong, as documented), no error."""
    rng = np.random.default_rng(5)
    A, W = packed(ilw, values(rng, 64, 96)), packed(ilw, rng.standard_normal((4, 40, 96)))
    for off in ([0, 1 << 30, 5, -7, 64], [-5, 70, 80, 90, 1 << 31 - 1], [60, 50, 40, 30, 20]):
        out = torch.full((66, 40), 9.0, device="cuda")
        ilw.mx_grouped_linear(A, W, torch.tensor(off, dtype=torch.int64).clamp(-(1 << 31), (1 << 31) - 1).int().cuda(), out=out[1:65])
        torch.cuda.synchronize()
        assert (out[0] == 9).all() and (out[65] == 9).all()
    ilw.device_status()


def test_products_follow_their_stream_and_graphs(ilw):
    """A chain on a side stream, and the same chain replayed from a graph on new inputs."""
    rng = np.random.default_rng(6)
    W = packed(ilw, rng.standard_normal((200, 256)) / 16)
    x = torch.from_numpy(rng.standard_normal((50, 256))).float().cuda()
    want = ilw.mx_linear(ilw.mx_quantize(x), W)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ilw.mx_linear(ilw.mx_quantize(x), W)
    side.synchronize()
    assert torch.equal(got, want)
    g = ilw.Graphed(lambda: ilw.mx_linear(ilw.mx_quantize(x), W))
    x.mul_(-3)
    want = ilw.mx_linear(ilw.mx_quantize(x), W)
    assert torch.equal(g.replay(), want)


def test_product_gives_up_a_bounded_wait(ilw):
    """A load that never comes: the kernel latches the status and returns, and the next call is right."""
    rng = np.random.default_rng(7)
    A, W = packed(ilw, values(rng, 300, 2048)), packed(ilw, rng.standard_normal((256, 2048)) / 45)
    few = ilw.MxTensor(A.codes[:4], A.scales[:4], A.k)
    want, want_few = ilw.mx_linear(A, W), ilw.mx_linear(few, W)
    short = packed(ilw, values(rng, 300, 512)), packed(ilw, rng.standard_normal((256, 512)) / 22)
    cases = ((A, W, want), (few, W, want_few), (*short, ilw.mx_linear(*short)))  # clusters on a tile, and one CTA (K = 512)
    for m, W, w in cases:
        assert ilw.lib().ilwdetr_debug_gemm_wait(0, 20_000_000) == 0  # (each CTA's first load)
        try:
            ilw.mx_linear(m, W)
            with pytest.raises(ilw.IlwError, match="wait"):
                ilw.device_status()
        finally:
            assert ilw.lib().ilwdetr_debug_gemm_wait(-1, 0) == 0
        assert torch.equal(ilw.mx_linear(m, W), w)
        ilw.device_status()


@pytest.mark.parametrize("M,N,K", [(4, 256, 8192), (3001, 1700, 4096)], ids=["cluster", "pair"])
def test_product_of_clusters_gives_up_a_bounded_wait(ilw, M, N, K):
    rng = np.random.default_rng(8)
    A, W = packed(ilw, values(rng, M, K)), packed(ilw, rng.standard_normal((N, K)) / np.sqrt(K))
    want = ilw.mx_linear(A, W)
    assert ilw.lib().ilwdetr_debug_gemm_wait(0, 20_000_000) == 0
    try:
        ilw.mx_linear(A, W)
        with pytest.raises(ilw.IlwError, match="wait"):
            ilw.device_status()
    finally:
        assert ilw.lib().ilwdetr_debug_gemm_wait(-1, 0) == 0
    assert torch.equal(ilw.mx_linear(A, W), want)
    ilw.device_status()


# ---------------------------------------------------------------------------- routing and combination
def ref_route(x, k, renormalize):
    """float64 x [T, E] -> expert, weight, offsets, source, slot."""
    T, E = x.shape
    x = np.where(np.isnan(x), -np.inf, x)
    expert, weight = np.full((T, k), -1), np.zeros((T, k))
    for t in range(T):
        order = np.argsort(-x[t], kind="stable")[:k]
        order = order[x[t, order] > -np.inf]
        if not len(order):
            continue
        p = np.exp(x[t] - x[t].max())
        expert[t, : len(order)] = order
        weight[t, : len(order)] = p[order] / (p[order].sum() if renormalize else p.sum())
    entries = sorted((expert[t, j], t, j) for t in range(T) for j in range(k) if expert[t, j] >= 0)
    offsets = np.searchsorted([e for e, _, _ in entries], np.arange(E + 1))
    source, slot = np.full(T * k, -1), np.full((T, k), -1)
    for s, (_, t, j) in enumerate(entries):
        source[s], slot[t, j] = t, s
    return expert, weight, offsets, source, slot


@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 8, 2), (7, 33, 4), (33, 64, 8), (300, 129, 6), (1000, 512, 16), (5000, 16, 1), (40000, 5, 2)])
def test_route_matches_64_bits(ilw, T, E, k, dtype, renormalize):
    """Many equal logits (a coarse grid), masked experts, whole rows masked, NaN."""
    rng = np.random.default_rng(T + E + k)
    x = np.round(rng.standard_normal((T, E)) * 4) / 4
    x[rng.random((T, E)) < 0.1] = -np.inf
    x[rng.random((T, E)) < 0.02] = np.nan
    x[rng.random(T) < 0.1] = -np.inf
    wide = torch.from_numpy(np.pad(x, ((0, 0), (1, 2)))).to(dtype).cuda()
    r = ilw.moe_route(wide[:, 1: 1 + E], k, renormalize)
    expert, weight, offsets, source, slot = ref_route(x, k, renormalize)
    for got, want in ((r.expert, expert), (r.offsets, offsets), (r.source, source), (r.slot, slot)):
        assert np.array_equal(got.cpu().numpy(), want)
    # exp's arguments are exact (a quarter grid); a sum of at most 512 terms and a quotient of fp32 exponentials of 2 ulp
    assert (np.abs(r.weight.double().cpu().numpy() - weight) <= (E + 8) * 2.0**-23 * weight).all()


@pytest.mark.parametrize("T", [1, 8, 111, 112, 113, 224, 225, 256, 257])
def test_route_of_few_tokens(ilw, T):
    """Either side of where one CTA does all."""
    rng = np.random.default_rng(T)
    for E in (8, 128, 256):
        x = np.round(rng.standard_normal((T, E)) * 4) / 4
        x[rng.random((T, E)) < 0.2] = -np.inf
        r = ilw.moe_route(torch.from_numpy(x).float().cuda(), 5, True)
        expert, weight, offsets, source, slot = ref_route(x, 5, True)
        for got, want in ((r.expert, expert), (r.offsets, offsets), (r.source, source), (r.slot, slot)):
            assert (got.cpu().numpy() == want).all()
        assert (np.abs(r.weight.double().cpu().numpy() - weight) <= (E + 8) * 2.0**-23 * weight).all()


@pytest.mark.parametrize("T", [100, 3000])
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_weights_of_logits_far_apart(ilw, T, renormalize):
    """Logits on a quarter grid, so that the exponentials' arguments are exact: of up to -80, each off by 2 ulp at most; a sum of
    8 of them and a quotient as above."""
    rng = np.random.default_rng(T)
    x = -rng.integers(0, 321, (T, 8)) / 4
    r = ilw.moe_route(torch.from_numpy(x).float().cuda(), 8, renormalize)
    expert, weight, *_ = ref_route(x, 8, renormalize)
    assert np.array_equal(r.expert.cpu().numpy(), expert)
    assert (np.abs(r.weight.double().cpu().numpy() - weight) <= (8 + 8) * 2.0**-23 * weight).all()


@pytest.mark.parametrize("T,E,k", [(4000, 256, 8), (4000, 64, 8), (20000, 128, 4), (200, 64, 16)])
@pytest.mark.parametrize("renormalize", [True, False])
def test_route_weights_as_exact_as_plain_operations(ilw, T, E, k, renormalize):
    """In norm, over many weights, no further from 64 bits than plain fp32 operations are (a tenth more for chance)."""
    x = 2 * torch.randn((T, E), device="cuda", generator=torch.Generator("cuda").manual_seed(T + E))
    r = ilw.moe_route(x, k, renormalize)

    def weights(x):
        top = torch.gather(x, 1, r.expert.long())
        p = torch.exp(x - top[:, :1])
        q = torch.exp(top - top[:, :1])
        return q / (q if renormalize else p).sum(1, keepdim=True)

    want = weights(x.double())
    assert (r.weight.double() - want).norm() <= 1.1 * (weights(x).double() - want).norm()


def test_route_of_many_experts_after_few(ilw):
    x = torch.randn(600, 256, device="cuda")
    first = ilw.moe_route(x, 3)
    ilw.moe_route(torch.randn(600, 8, device="cuda"), 3)
    assert all(torch.equal(a, b) for a, b in zip(ilw.moe_route(x, 3), first))


def test_route_extremes(ilw):
    big = float(np.float32(3.4028234e38))
    x = torch.tensor([[big, -big, 0.0, -0.0], [-big, -big, -big, float("-inf")], [0.0, -0.0, -0.0, 0.0], [float("nan")] * 4,
                      [float("inf"), 1.0, 2.0, 3.0]])
    r = ilw.moe_route(x.cuda(), 3)
    assert r.expert.tolist() == [[0, 2, 3], [0, 1, 2], [0, 1, 2], [-1, -1, -1], [0, 3, 2]]
    w = r.weight.cpu()
    assert w[0].tolist() == [1, 0, 0] and torch.allclose(w[1:3], torch.full((2, 3), 1 / 3)) and (w[3] == 0).all() and w[4].isnan().all()
    empty = ilw.moe_route(torch.empty((0, 6), device="cuda"), 2)
    assert empty.offsets.tolist() == [0] * 7 and empty.expert.shape == (0, 2)


def test_route_refuses_a_huge_k_before_it_makes_room(ilw):
    x = torch.randn(2000, 8, device="cuda")
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    for k in (0, -3, 9, 17, 1 << 26, (1 << 31) - 1):
        with pytest.raises(ilw.IlwError, match="moe_route"):
            ilw.moe_route(x, k)
    assert torch.cuda.max_memory_allocated() - before < 1 << 20


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (5, 2, 33), (64, 8, 256), (300, 3, 1000), (17, 16, 40)])
@pytest.mark.parametrize("residual", [False, True])
def test_combine_matches_64_bits(ilw, T, k, N, dtype, residual):
    rng = np.random.default_rng(T + k + N)
    R = T * k + 3
    Y = torch.from_numpy(rng.standard_normal((R, N + 8))).to(dtype).cuda()[:, 8:]
    Y[T * k:] = float("nan")  # rows that no slot names
    slot = rng.permutation(T * k).reshape(T, k).astype(np.int32)
    slot[rng.random((T, k)) < 0.2] = -1
    w = rng.random((T, k)).astype(np.float32)
    res = torch.from_numpy(rng.standard_normal((T, N))).to(dtype).cuda() if residual else None
    got = ilw.moe_combine(Y, torch.from_numpy(slot).cuda(), torch.from_numpy(w).cuda(), residual=res)
    y = np.where(slot[..., None] < 0, 0, Y.double().cpu().numpy()[slot]) * w[..., None]
    want, mass = y.sum(1), np.abs(y).sum(1)
    if residual:
        want, mass = want + res.double().cpu().numpy(), mass + np.abs(res.double().cpu().numpy())
    tol = (k + 1) * 2.0**-24 * mass + EPS[dtype] * (np.abs(want) + (k + 1) * 2.0**-24 * mass) + (2.0**-25 if dtype == torch.float16 else 0)
    assert got.dtype == dtype and (np.abs(got.double().cpu().numpy() - want) <= tol).all()
    if residual:
        ilw.moe_combine(Y, torch.from_numpy(slot).cuda(), torch.from_numpy(w).cuda(), residual=res, out=res)
        assert torch.equal(res, got)


def test_combine_reports_a_bad_slot(ilw):
    Y = torch.ones((4, 8), device="cuda")
    out = ilw.moe_combine(Y, torch.tensor([[0, 4], [-2, 1]], dtype=torch.int32, device="cuda"), torch.ones((2, 2), device="cuda"))
    assert (out == 1).all()
    with pytest.raises(ilw.IlwError, match="index"):
        ilw.device_status()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_combine_of_a_row_past_2_30(ilw, dtype):
    """Rows of more than 2^30 values off 16-byte boundaries: a column counter stepped by a row passes 2^31."""
    N = 2**30 + 9
    Y = (torch.arange(N, dtype=torch.int32, device="cuda") % 251).to(dtype)[None]
    slot = torch.tensor([[0, -1], [0, 0]], dtype=torch.int32, device="cuda")
    out = torch.full((3, N), -1.0, dtype=dtype, device="cuda")
    ilw.moe_combine(Y, slot, torch.ones((2, 2), device="cuda"), out=out[1:])  # (whole numbers up to 500: exact)
    assert (out[0] == -1).all() and torch.equal(out[1], Y[0]) and torch.equal(out[2], 2 * Y[0])
    ilw.device_status()


def test_combine_of_almost_2_31_tokens(ilw):
    """As many tokens as are accepted: a token counter stepped by the grid's height passes 2^31."""
    T = 2**31 - 1
    slot = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    slot[-3:, 0] = torch.tensor([1, -1, 1], device="cuda")
    Y = torch.tensor([[1.0], [2.0]], dtype=torch.bfloat16, device="cuda")
    out = torch.full((T + 2, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    ilw.moe_combine(Y, slot, torch.ones((T, 1), device="cuda"), out=out[1:-1])
    assert out[-5:, 0].tolist() == [1, 2, 0, 2, 7] and out[0, 0] == 7 and bool((out[1:-4] == 1).all())
    ilw.device_status()


# ---------------------------------------------------------------------------- the feed-forward
@pytest.mark.parametrize("act,dtype", [("silu_gate", torch.bfloat16), ("gelu", torch.float32), ("silu_gate", torch.float16)])
@pytest.mark.parametrize("T", [0, 1, 37, 600])
def test_experts_feed_forward(ilw, T, act, dtype):
    """Each step against 64 bits on what the step before it gave (a rounding that falls the other way before the second
    quantisation would otherwise be a whole code)."""
    rng = np.random.default_rng(T)
    E, d, F, top = 6, 192, 320, 2
    F1 = 2 * F if act == "silu_gate" else F
    w1 = torch.from_numpy(rng.standard_normal((E, F1, d)) / np.sqrt(d)).float().cuda()
    w2 = torch.from_numpy(rng.standard_normal((E, d, F)) / np.sqrt(F)).float().cuda()
    if act == "silu_gate":
        assert torch.equal(ilw.gate_rows(w1[:, :F], w1[:, F:])[:, 1::2], w1[:, F:])
        w1 = ilw.gate_rows(w1[:, :F], w1[:, F:])
    b1 = torch.from_numpy(0.1 * rng.standard_normal((E, F1))).float().cuda()
    ffn = ilw.MxExperts(w1, w2, top, act=act, b1=b1)
    x = torch.from_numpy(rng.standard_normal((T, d))).to(dtype).cuda()
    logits = torch.from_numpy(rng.standard_normal((T, E))).to(dtype).cuda()
    logits[T // 2:, 1:] = float("-inf")  # half of the tokens have one expert left
    got = ffn.forward(x, logits, residual=x)
    assert got.dtype == dtype and got.shape == (T, d)
    if not T:
        return
    r = ilw.moe_route(logits, top)
    expert, weight, offsets, source, slot = ref_route(logits.double().cpu().numpy(), top, True)
    assert np.array_equal(r.source.cpu().numpy(), source) and np.array_equal(r.offsets.cpu().numpy(), offsets)
    a = ilw.mx_quantize(x, gather=r.source)
    h = ilw.mx_grouped_linear(a, ffn.w1, r.offsets, bias=b1, act=act, out_dtype=dtype)
    q = ilw.mx_quantize(h)
    y = ilw.mx_grouped_linear(q, ffn.w2, r.offsets, out_dtype=dtype)
    av, qv = ref_values(*host(a), d), ref_values(*host(q), F)
    w1v, w2v = ref_values(*host(ffn.w1), d), ref_values(*host(ffn.w2), F)
    xv = np.where(source[:, None] < 0, 0, x.double().cpu().numpy()[source])
    assert np.array_equal(av, ref_values(*[p.astype(np.uint8) for p in _bytes(*ref_quantize(xv))], d))
    for e in range(E):
        s = slice(int(offsets[e]), int(offsets[e + 1]))
        if s.stop > s.start:
            check_product(h[s], av[s], w1v[e], b1[e].double().cpu().numpy(), act, dtype)
            check_product(y[s], qv[s], w2v[e], None, "none", dtype)
    assert torch.equal(got, ilw.moe_combine(y, r.slot, r.weight, residual=x))
    ilw.device_status()


@pytest.mark.parametrize("E", [1, 3])
def test_gated_products_with_gate_and_up_biases_given_apart(ilw, E):
    """Weights and biases of the gates and of what they gate, joined by gate_rows: each column takes its own bias."""
    rng = np.random.default_rng(E)
    counts, F, K = [40, 0, 9][:E], 50, 96
    off = np.r_[0, np.cumsum(counts)]
    gate, up = (torch.from_numpy(rng.standard_normal((E, F, K)) / np.sqrt(K)) for _ in range(2))
    bg, bu = (torch.from_numpy(rng.standard_normal((E, F))).float() for _ in range(2))
    A, W = packed(ilw, values(rng, int(off[-1]), K)), packed(ilw, ilw.gate_rows(gate, up).numpy())
    a, w = ref_values(*host(A), K), ref_values(*host(W), K)
    b = np.zeros((E, 2 * F))
    b[:, 0::2], b[:, 1::2] = bg.numpy(), bu.numpy()
    got = ilw.mx_grouped_linear(A, W, torch.from_numpy(off.astype(np.int32)).cuda(), ilw.gate_rows(bg, bu, dim=1).cuda(), act="silu_gate",
                                out_dtype=torch.bfloat16)
    for e in range(E):
        if counts[e]:
            check_product(got[off[e]: off[e + 1]], a[off[e]: off[e + 1]], w[e], b[e], "silu_gate", torch.bfloat16)
    one = ilw.MxTensor(W.codes[0], W.scales[0], K)
    first = ilw.mx_linear(ilw.MxTensor(A.codes[:40], A.scales[:40], K), one, ilw.gate_rows(bg[0], bu[0]).cuda(), act="silu_gate", out_dtype=torch.float32)
    check_product(first, a[:40], w[0], b[0], "silu_gate", torch.float32)


def _bytes(code, byte):
    return code[:, 0::2] | code[:, 1::2] << 4, byte
