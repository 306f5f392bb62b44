"""Int8 operators with float scales on the GPU against plain restatements in 64 bits.

Codes are those of the exact quotient and scales correctly rounded, so quantising is exact.  Products: the sum of code products is
exact below 2^24, and past that of fp32 additions of at most 2^-23 of the sum of magnitudes each (one for 16 of K, and a few
to join parts); scaling it by two factors takes three roundings, the bias one.  The activations have a slope of at most 1.13 (GELU)
and take at most 8 further roundings, and the output is rounded once to its type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

FLOATS = [torch.float32, torch.float16, torch.bfloat16]
EPS = {torch.float32: 2.0**-24, torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8}  # half an ulp, relative


@pytest.fixture(scope="module")
def ilw():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2607_24981_gb300 as m
    from paper_2607_24981_gb300 import build

    build.build()
    m.lib()
    return m


def generator(seed):
    return torch.Generator("cuda").manual_seed(seed)


# ---------------------------------------------------------------------------- restatements
def ref_quantize(x):
    """Codes and scales of float64 rows x [R, K] (on any device)."""
    amax = x.abs().amax(1)
    fine = torch.isfinite(x).all(1)
    scale = torch.where(amax > 0, (amax / 127).float().double().clamp(min=2.0**-126), 0.0)
    code = torch.round(x / scale[:, None])  # (a quotient of two fp32 numbers is no closer than 2^-33 of itself to a half that it is not)
    code = torch.where((fine & (amax > 0))[:, None], code, 0.0)
    return code.to(torch.int8), torch.where(fine, scale, torch.nan).float()


def made(ilw, seed, R, K, weights=False):
    """Weights, or activations in rows of different sizes, as int8 (by the restatement)."""
    x = torch.randn((R, K), generator=generator(seed), device="cuda")
    x = x / K**0.5 if weights else x * torch.exp2(torch.randint(-6, 4, (R, 1), generator=generator(seed + 1), device="cuda").float())
    if not weights and R > 4:
        x[R // 3] = 0
    out = ilw.i8_empty(R, K)
    code, scale = ref_quantize(x.double())
    out.codes.copy_(code)
    out.scales.copy_(scale)
    return out


def check_product(got, A, W, bias, act):
    """got [M, n] against the 64-bit product of int8 A and W; the bound of the module's docstring."""
    a, w, sa, sw = A.codes.double(), W.codes.double(), A.scales.double()[:, None], W.scales.double()
    K = a.shape[1]
    mass = a.abs() @ w.abs().T
    z, tol = a @ w.T * sa * sw, torch.where(mass >= 2.0**24, (K / 16 + 16) * 2.0**-23 * mass, 0.0) * sa * sw
    tol = tol + 3 * 2.0**-24 * (z.abs() + tol)
    if bias is not None:
        z = z + bias.double()
        tol = tol + 2.0**-24 * (z.abs() + tol)
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
    tol = tol + EPS[got.dtype] * (want.abs() + tol) + (2.0**-25 if got.dtype == torch.float16 else 1e-44)  # (half a subnormal's step)
    err = (got.double() - want).abs()
    assert got.shape == want.shape and (err <= tol).all(), f"{int((err > tol).sum())} of {err.numel()} outside, worst {float((err / tol).max()):.3g} times the bound"


# ---------------------------------------------------------------------------- quantisation
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("R,K", [(1, 1), (3, 31), (2, 32), (5, 33), (4, 264), (7, 257), (2, 2051), (130, 520), (3, 2048), (3, 4096), (2, 4097), (2, 8200),
                                 (2, 16384), (1, 40000), (2, 20007)])
def test_quantize_matches_64_bits(ilw, dtype, R, K):
    x = torch.randn((R, K), generator=generator(K), device="cuda") * torch.exp2(torch.randint(-12, 12, (R, 1), generator=generator(R), device="cuda").float())
    x[:, K // 2] *= 7
    if R > 2:
        x[1] = 0
    x = x.to(dtype)
    got = ilw.i8_quantize(x)
    code, scale = ref_quantize(x.double())
    assert got.codes.dtype == torch.int8 and got.codes.shape == (R, K) and got.codes.stride(0) % 16 == 0
    assert torch.equal(got.codes, code) and torch.equal(got.scales, scale)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("K", [256, 253])
def test_quantize_halves_and_their_neighbours(ilw, dtype, K):
    """Quotients that are halves exactly, and the fp32 numbers next to them, for scales of which the reciprocal is rounded."""
    rows = []
    for s in (1.0, 0.75, 3.0, 1 / 128, 0.0078125 * 5, 2.0**-126, 2.0**119):
        n = torch.arange(K, dtype=torch.float64) - K // 2
        half = ((n.clamp(-126, 125) + 0.5) * s).float()
        for shift in (0, 1, -1):
            v = (half.view(torch.int32) + shift).view(torch.float32).to(dtype).float()
            v[0] = 127 * s
            rows.append(v)
    x = torch.stack(rows)[:, :K].cuda()
    x = torch.where(torch.isfinite(x.to(dtype)), x, 0.0).to(dtype)
    got, (code, scale) = ilw.i8_quantize(x), ref_quantize(x.double())
    assert torch.equal(got.codes, code) and torch.equal(got.scales, scale)
    if dtype == torch.float32:
        odd = (x.double() / scale.double()[:, None]).remainder(1) == 0.5
        assert int(odd.sum()) > 100 and bool((got.codes[odd] % 2 == 0).all())


@pytest.mark.parametrize("dtype,digits", [(torch.float16, 10), (torch.bfloat16, 7)])
@pytest.mark.parametrize("exponent", [0, 5, -9])
def test_quantize_every_pair_of_significands(ilw, dtype, digits, exponent):
    """Every largest value of a binade (a row each) with every smaller value down to 1/256 of the binade, of both signs."""
    n = 1 << digits
    largest = (1 + torch.arange(n, device="cuda", dtype=torch.float64) / n) * 2.0**exponent
    values = torch.cat([largest * 2.0**-b for b in range(9)])
    x = torch.minimum(values[None, :], largest[:, None]) * torch.where(torch.arange(len(values), device="cuda") % 3 == 1, -1.0, 1.0)
    x[:, 0] = largest
    q = ilw.i8_quantize(x.to(dtype))
    for rows in torch.arange(n, device="cuda").split(128):
        code, scale = ref_quantize(x[rows].to(dtype).double())
        assert torch.equal(q.scales[rows], scale) and torch.equal(q.codes[rows], code)


def test_quantize_special_values(ilw):
    """Rows of zeros, subnormals, the largest numbers, infinities and NaN."""
    big, inf, nan = 3.4028234e38, float("inf"), float("nan")
    x = torch.zeros((8, 40))
    x[1, 3], x[1, 5] = 1e-45, -3e-45
    x[2, 0], x[2, 1] = big, -big
    x[3, 7] = inf
    x[4, 7] = -inf
    x[5, 39] = nan
    x[6, 0], x[6, 1], x[6, 2] = 127 * 2.0**-126, -(2.0**-127), 2.0**-126
    x[7] = -0.0
    for y in (x, x[:, :33].contiguous(), torch.cat([x[:, :39], torch.zeros(8, 5000), x[:, 39:]], 1)):
        got = ilw.i8_quantize(y.cuda())
        code, scale = ref_quantize(y.double().nan_to_num(nan=nan, posinf=inf, neginf=-inf))
        assert torch.equal(got.codes.cpu(), code)
        assert torch.equal(got.scales.cpu().nan_to_num(nan=-1.0), scale.nan_to_num(nan=-1.0))
        values = ilw.i8_dequantize(got)
        assert bool(values[0].eq(0).all()) and bool(values[3].isnan().all()) and bool(values[4].isnan().all()) and bool(values[5].isnan().all()) == (y.shape[1] > 33)


def test_quantize_gathers_rows(ilw):
    x = torch.randn((50, 100), generator=generator(1), device="cuda")
    at = torch.tensor([3, 3, -1, 49, 0, -1, 7], dtype=torch.int32, device="cuda")
    got = ilw.i8_quantize(x, gather=at)
    want = ilw.i8_quantize(torch.where(at[:, None] >= 0, x[at.long().clamp(min=0)], 0.0))
    assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales)
    ilw.device_status()
    bad = ilw.i8_quantize(x, gather=torch.tensor([1, 50, -2], dtype=torch.int32, device="cuda"))
    assert torch.equal(bad.codes[0], ilw.i8_quantize(x[1:2]).codes[0]) and bool((bad.codes[1:] == 0).all()) and bool((bad.scales[1:] == 0).all())
    with pytest.raises(ilw.IlwError, match="index"):
        ilw.device_status()
    none = ilw.i8_quantize(x, gather=torch.empty(0, dtype=torch.int32, device="cuda"))
    assert none.codes.shape == (0, 100) and none.scales.shape == (0,)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("K", [96, 101])
def test_quantize_rows_with_strides_and_offsets(ilw, dtype, K):
    """Rows at any element, and a result among other memory, which stays as it was."""
    wide = torch.randn((9, 150), generator=generator(K), device="cuda").to(dtype)
    for shift in (0, 1, 3, 8):
        x = wide[:, shift: shift + K]
        codes = torch.full((9, 160), 77, dtype=torch.int8, device="cuda")
        scales = torch.full((11,), 5.0, device="cuda")
        out = ilw.I8Tensor(codes[:, 16: 16 + K], scales[1:10])
        assert ilw.i8_quantize(x, out=out) is out
        code, scale = ref_quantize(x.double())
        assert torch.equal(out.codes, code) and torch.equal(out.scales, scale)
        codes[:, 16: 16 + K] = 77
        assert bool((codes == 77).all()) and scales[0] == 5 and scales[-1] == 5


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("K", [256, 251, 17, 1])
def test_dequantize_every_code(ilw, dtype, K):
    scales = torch.tensor([1.0, 0.0, 2.0**-126, 3e-5, 7.3, 2.6e36, 2e38, float("nan")], device="cuda")
    m = ilw.i8_empty(8, K)
    m.codes.copy_((torch.arange(K, device="cuda") - 128).to(torch.int8).expand(8, K))
    m.scales.copy_(scales)
    want = (m.codes.float() * scales[:, None]).to(dtype)
    wide = torch.full((8, K + 9), 3.0, device="cuda", dtype=dtype)
    for out in (None, wide[:, 8: 8 + K], wide[:, 3: 3 + K]):
        wide.fill_(3.0)
        got = ilw.i8_dequantize(m, dtype=dtype, out=out)
        assert got.dtype == dtype and torch.equal(got.float().nan_to_num(nan=-0.123), want.float().nan_to_num(nan=-0.123))
        if out is not None:
            out.fill_(3.0)
            assert bool((wide == 3.0).all())


# ---------------------------------------------------------------------------- products
@pytest.mark.parametrize("act,bias", [("none", False), ("none", True), ("gelu", True), ("silu_gate", False), ("silu_gate", True)])
@pytest.mark.parametrize("M,N,K", [(1, 2, 1), (1, 128, 4096), (3, 130, 512), (2, 66, 15), (5, 64, 16), (8, 300, 17), (9, 130, 100), (16, 300, 33), (17, 128, 250),
                                   (33, 1000, 2048), (64, 256, 1000), (129, 258, 65), (200, 514, 640), (300, 1002, 1030), (1000, 384, 1536)])
def test_linear_matches_64_bits(ilw, M, N, K, act, bias):
    A, W = made(ilw, 1, M, K), made(ilw, 3, N, K, weights=True)
    b = torch.randn(N, device="cuda", generator=generator(5)) if bias else None
    for dtype in FLOATS:
        got = ilw.i8_linear(A, W, b, act=act, out_dtype=dtype)
        assert got.dtype == dtype
        check_product(got, A, W, b, act)
    assert torch.equal(got, ilw.i8_linear(A, W, b, act=act, out_dtype=dtype))
    ilw.device_status()


@pytest.mark.parametrize("M", [1, 8, 40, 400])
@pytest.mark.parametrize("code", [127, -128])
@pytest.mark.parametrize("K", [1024, 1030, 8192, (1 << 17) - 1])
def test_linear_of_the_largest_codes(ilw, M, code, K):
    """Sums past 2^24, and up to K = 1024 (2^24 itself) exact ones."""
    A, W = ilw.i8_empty(M, K), ilw.i8_empty(130, K)
    for m in (A, W):
        m.codes.fill_(code)
        m.scales.fill_(1.0)
    A.codes[:, 1] = 1
    got = ilw.i8_linear(A, W, out_dtype=torch.float32)
    want = A.codes.double() @ W.codes.double().T
    if K <= 1024:
        assert torch.equal(got.double(), want)
    check_product(got, A, W, None, "none")


def test_linear_scales_and_nan(ilw):
    """A row or channel of scale NaN is NaN, of scale 0 is the bias; tiny and huge scales meet without overflow where the result fits."""
    A, W = made(ilw, 1, 12, 256), made(ilw, 3, 40, 256, weights=True)
    A.scales[2], A.scales[3], W.scales[5], W.scales[7] = float("nan"), 0.0, float("nan"), 0.0
    A.scales[4], W.scales[9] = 1e-30, 1e28
    b = torch.randn(40, device="cuda", generator=generator(5))
    got = ilw.i8_linear(A, W, b, out_dtype=torch.float32)
    nan = torch.zeros((12, 40), dtype=torch.bool, device="cuda")
    nan[2], nan[:, 5] = True, True
    assert torch.equal(got.isnan(), nan)
    assert torch.equal(got[3][~nan[3]], b[~nan[3]]) and torch.equal(got[:, 7][~nan[:, 7]], b[7].expand(11))
    keep, cols = [i for i in range(12) if i != 2], [i for i in range(40) if i != 5]
    check_product(got[keep][:, cols], ilw.I8Tensor(A.codes[keep], A.scales[keep]), ilw.I8Tensor(W.codes[cols], W.scales[cols]), b[cols], "none")


@pytest.mark.parametrize("M", [3, 150])
def test_linear_rows_with_strides(ilw, M):
    """Operands and results that are parts of larger tensors: what is around the codes is not read, around the result not written."""
    N, K = 260, 250
    A, W = made(ilw, 1, M, K), made(ilw, 3, N, K, weights=True)
    b = torch.randn(N, device="cuda", generator=generator(5))
    ac = torch.full((M, 320), -128, dtype=torch.int8, device="cuda")[:, 32: 32 + K]
    wc = torch.full((N, 272), 127, dtype=torch.int8, device="cuda")[:, 16: 16 + K]
    ac.copy_(A.codes)
    wc.copy_(W.codes)
    want = ilw.i8_linear(A, W, b, act="gelu")
    for shift in (0, 3, 8):
        wide = torch.full((M, N + 20), 9.0, dtype=torch.bfloat16, device="cuda")
        ilw.i8_linear(ilw.I8Tensor(ac, A.scales), ilw.I8Tensor(wc, W.scales), b, act="gelu", out=wide[:, shift: shift + N])
        assert torch.equal(wide[:, shift: shift + N], want)
        wide[:, shift: shift + N] = 9.0
        assert bool((wide == 9).all())
    ilw.device_status()


def test_linear_of_nothing(ilw):
    A, W = made(ilw, 1, 4, 64), made(ilw, 3, 10, 64, weights=True)
    assert ilw.i8_linear(ilw.I8Tensor(A.codes[:0], A.scales[:0]), W).shape == (0, 10)
    assert ilw.i8_linear(A, ilw.I8Tensor(W.codes[:0], W.scales[:0])).shape == (4, 0)


GROUPS = {"few": [1, 0, 2, 9, 0, 3], "ragged": [130, 0, 1, 257, 16, 64, 0], "one": [0, 0, 300, 0], "none": [0, 0, 0], "single": [50], "even": [32] * 16, "many": [5, 0, 1] * 43,
          "long": [700, 0, 1, 333, 1024, 225, 95]}


@pytest.mark.parametrize("counts", GROUPS.values(), ids=GROUPS.keys())
@pytest.mark.parametrize("N,K,act", [(130, 100, "none"), (256, 1536, "silu_gate"), (66, 544, "gelu"), (1001, 250, "none")])
def test_grouped_matches_64_bits(ilw, counts, N, K, act):
    off, E = np.r_[0, np.cumsum(counts)], len(counts)
    M = int(off[-1])
    A, W = made(ilw, 1, M, K), made(ilw, 3, E * N, K, weights=True)
    W = ilw.I8Tensor(W.codes.unflatten(0, (E, N)), W.scales.view(E, N))
    b = torch.randn((E, N), device="cuda", generator=generator(5))
    offsets = torch.from_numpy(off.astype(np.int32)).cuda()
    for dtype in FLOATS[:: 2 if M > 1000 else 1]:
        got = ilw.i8_grouped_linear(A, W, offsets, b, act=act, out_dtype=dtype)
        for e in range(E):
            s = slice(int(off[e]), int(off[e + 1]))
            if counts[e]:
                check_product(got[s], ilw.I8Tensor(A.codes[s], A.scales[s]), ilw.I8Tensor(W.codes[e], W.scales[e]), b[e], act)
    ilw.device_status()


def test_grouped_leaves_zeros_where_no_expert_is(ilw):
    """Offsets that begin past 0 and end before M; ones out of order or range reach nothing outside."""
    A, W = made(ilw, 1, 600, 64), made(ilw, 3, 4 * 34, 64, weights=True)
    W = ilw.I8Tensor(W.codes.unflatten(0, (4, 34)), W.scales.view(4, 34))
    for lo, hi in ((5, 9), (5, 590), (0, 0), (600, 600)):
        offsets = torch.tensor([lo, lo, (lo + hi) // 2, hi, hi], dtype=torch.int32, device="cuda")
        out = torch.full((600, 34), 7.0, device="cuda")
        ilw.i8_grouped_linear(A, W, offsets, out=out)
        assert bool((out[:lo] == 0).all()) and bool((out[hi:] == 0).all())
        for e, (a, z) in enumerate(((lo, lo), (lo, (lo + hi) // 2), ((lo + hi) // 2, hi))):
            if z > a:
                check_product(out[a:z], ilw.I8Tensor(A.codes[a:z], A.scales[a:z]), ilw.I8Tensor(W.codes[e], W.scales[e]), None, "none")
    for offsets in ([50, 20, 70, 10, 60], [-5, 3, 1 << 30, 2, 5], [0, 1 << 31 - 1, -(1 << 31), 600, 600], [600, 0, 600, 0, 600]):
        wide = torch.full((620, 34), 7.0, device="cuda")
        ilw.i8_grouped_linear(A, W, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=wide[10:610])
        assert bool((wide[:10] == 7).all()) and bool((wide[610:] == 7).all())
    ilw.device_status()


def test_grouped_of_very_many_experts(ilw):
    E, N, K = 1024, 40, 48
    counts = torch.randint(0, 3, (E,), generator=torch.Generator().manual_seed(1))
    off = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)])
    M = int(off[-1])
    A, W = made(ilw, 1, M, K), made(ilw, 3, E * N, K, weights=True)
    W = ilw.I8Tensor(W.codes.unflatten(0, (E, N)), W.scales.view(E, N))
    got = ilw.i8_grouped_linear(A, W, off.int().cuda(), out_dtype=torch.float32)
    expert = torch.repeat_interleave(torch.arange(E), counts).cuda()
    z = torch.einsum("mk,mnk->mn", A.codes.double(), W.codes.double()[expert]) * A.scales.double()[:, None] * W.scales.double()[expert]
    assert bool(((got.double() - z).abs() <= 4 * 2.0**-24 * z.abs()).all())
    one = ilw.i8_grouped_linear(ilw.I8Tensor(A.codes[:7], A.scales[:7]), ilw.I8Tensor(W.codes[:1], W.scales[:1]), torch.tensor([0, 7], dtype=torch.int32, device="cuda"))
    assert torch.equal(one, ilw.i8_linear(ilw.I8Tensor(A.codes[:7], A.scales[:7]), ilw.I8Tensor(W.codes[0], W.scales[0])))


@pytest.mark.parametrize("M", [2, 300])
def test_products_follow_their_stream_and_graphs(ilw, M):
    """On a stream that is not the default one, and captured into two graphs that are replayed in turn on new inputs."""
    N, K = 520, 600
    W = made(ilw, 3, N, K, weights=True)
    x = [torch.randn((M, K), generator=generator(i), device="cuda") for i in range(3)]
    want = [ilw.i8_linear(ilw.i8_quantize(v), W, act="gelu") for v in x]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        buf = torch.zeros_like(x[0])
        torch.cuda._sleep(2_000_000)
        buf.copy_(x[0])
        got = ilw.i8_linear(ilw.i8_quantize(buf), W, act="gelu")
    side.synchronize()
    assert torch.equal(got, want[0])
    graphs, outs, ins = [], [], []
    for _ in range(2):
        b = x[0].clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(ilw.i8_linear(ilw.i8_quantize(b), W, act="gelu"))
        graphs.append(g)
        ins.append(b)
    for i, j in ((1, 2), (2, 0), (0, 1)):
        ins[0].copy_(x[i])
        ins[1].copy_(x[j])
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[i]) and torch.equal(outs[1], want[j])
    ilw.device_status()


# ---------------------------------------------------------------------------- the feed-forward
@pytest.mark.parametrize("act,dtype", [("silu_gate", torch.bfloat16), ("gelu", torch.float32), ("silu_gate", torch.float16)])
@pytest.mark.parametrize("T", [0, 1, 37, 600, 2500])
def test_experts_feed_forward(ilw, T, act, dtype):
    """Routing by sigmoid scores, a bias and groups, rows gathered and quantised, both products, the join: each step against 64 bits on
    what the step before it gave."""
    E, d, F, top = 8, 192, 320, 2
    F1 = 2 * F if act == "silu_gate" else F
    gen = generator(T + 1)
    w1 = torch.randn((E, F1, d), generator=gen, device="cuda") / d**0.5
    w2 = torch.randn((E, d, F), generator=gen, device="cuda") / F**0.5
    b1, bias = 0.1 * torch.randn((E, F1), generator=gen, device="cuda"), 0.1 * torch.randn(E, generator=gen, device="cuda")
    how = dict(score="sigmoid", bias=bias, groups=4, top_groups=2, group_best=1, scale=2.0)
    ffn = ilw.I8Experts(w1, w2, top, act=act, b1=b1, **how)
    x = torch.randn((T, d), generator=gen, device="cuda").to(dtype)
    logits = torch.randn((T, E), generator=gen, device="cuda").to(dtype)
    logits[T // 2:, 1:] = float("-inf")  # half of the tokens have one expert left
    got = ffn.forward(x, logits, residual=x)
    assert got.dtype == dtype and got.shape == (T, d)
    if not T:
        return
    r = ilw.moe_route(logits, top, **how)
    off = r.offsets.tolist()
    a = ilw.i8_quantize(x, gather=r.source)
    code, scale = ref_quantize(torch.where(r.source[:, None] >= 0, x.double()[r.source.long().clamp(min=0)], 0.0))
    assert torch.equal(a.codes, code) and torch.equal(a.scales, scale)
    h = ilw.i8_grouped_linear(a, ffn.w1, r.offsets, bias=b1, act=act, out_dtype=dtype)
    q = ilw.i8_quantize(h)
    y = ilw.i8_grouped_linear(q, ffn.w2, r.offsets, out_dtype=dtype)
    for e in range(E):
        s = slice(off[e], off[e + 1])
        if s.stop > s.start:
            check_product(h[s], ilw.I8Tensor(a.codes[s], a.scales[s]), ilw.I8Tensor(ffn.w1.codes[e], ffn.w1.scales[e]), b1[e], act)
            check_product(y[s], ilw.I8Tensor(q.codes[s], q.scales[s]), ilw.I8Tensor(ffn.w2.codes[e], ffn.w2.scales[e]), None, "none")
    assert torch.equal(got, ilw.moe_combine(y, r.slot, r.weight, residual=x))
    ilw.device_status()


def test_experts_in_two_graphs(ilw):
    """Captured twice, replayed in turn on new inputs, some of whose tokens have no expert."""
    E, d, F, T = 16, 96, 160, 700
    gen = generator(5)
    ffn = ilw.I8Experts(torch.randn((E, 2 * F, d), generator=gen, device="cuda") / d**0.5, torch.randn((E, d, F), generator=gen, device="cuda") / F**0.5, 3,
                        score="sigmoid", bias=0.1 * torch.randn(E, generator=gen, device="cuda"), groups=4, top_groups=2)
    x = [torch.randn((T, d), generator=gen, device="cuda").half() for _ in range(3)]
    logits = [torch.randn((T, E), generator=gen, device="cuda") for _ in range(3)]
    for i, v in enumerate(logits):
        v[100 * i:200 * i] = float("-inf")
    want = [ffn.forward(a, b) for a, b in zip(x, logits)]
    graphs = []
    for _ in range(2):
        a, b, g = x[0].clone(), logits[0].clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = ffn.forward(a, b)
        graphs.append((a, b, g, y))
    for pair in ((1, 2), (2, 0), (0, 1)):
        for (a, b, g, y), i in zip(graphs, pair):
            a.copy_(x[i])
            b.copy_(logits[i])
            g.replay()
        torch.cuda.synchronize()
        for (a, b, g, y), i in zip(graphs, pair):
            assert torch.equal(y, want[i])
    assert bool((want[2][200:400] == 0).all())
    ilw.device_status()


# ---------------------------------------------------------------------------- every form of the products
def form_of(ilw, M, N, K, experts, act, dtype):
    """What the library takes for a product with contiguous operands on this GPU: "one" CTA a tile, "pair" of SMs, "few" tokens, or how many
    CTAs share a tile's K; and the tokens of a tile."""
    import ctypes

    from paper_2607_24981_gb300 import int8, mx

    got, ld, wide = (ctypes.c_int32 * 3)(), -(-K // 16) * 16, N // 2 if act == "silu_gate" else N
    y_form = {torch.float32: 232, torch.float16: 216, torch.bfloat16: 217}[dtype]
    rc = ilw.lib().ilwdetr_debug_i8_form(int8.gemm_struct(1 << 20, ld, 1 << 20, 1 << 20, ld, N * ld, 1 << 20, 0, 1 << 20 if experts else 0, M, N, K, experts or 1,
                                                          mx.ACTS[act], y_form, 1 << 20, wide), 0, got)
    assert rc == 0, ilw.lib().ilwdetr_last_error()
    return ["one", got[1], "pair", "few"][got[0]], got[2]


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("form,M,N,K,bias", [
    ("pair", 5000, 2600, 500, True), ("pair", 3001, 1712, 1030, False), ("pair", 3001, 514, 1030, True), ("pair", 700, 1000, 1030, False), ("pair", 200, 1712, 2100, True),
    ("pair", 1500, 1000, 4200, True), (2, 16, 5000, 8200, True), (2, 40, 5000, 4200, False), (2, 100, 5000, 4200, True), (4, 130, 1000, 2100, True), (4, 333, 514, 2100, False),
    (4, 700, 514, 4200, True), (8, 40, 1000, 8200, True), (8, 60, 1000, 4200, False), (8, 333, 130, 8200, True), ("one", 130, 1712, 500, True), ("one", 700, 1712, 200, False),
    ("one", 5000, 514, 200, True), ("few", 5, 1000, 500, True), ("few", 40, 260, 300, False), ("few", 8, 5000, 4200, True), ("few", 3, 34, 9000, True)])
def test_every_form_with_every_activation(ilw, form, M, N, K, bias, dtype):
    A, W = made(ilw, 1, M, K), made(ilw, 3, N, K, weights=True)
    b = torch.randn(N, device="cuda", generator=generator(5)) if bias else None
    for act in ("none", "gelu", "silu_gate"):
        assert form_of(ilw, M, N, K, None, act, dtype)[0] == form
        got = ilw.i8_linear(A, W, b, act=act, out_dtype=dtype)
        check_product(got, A, W, b, act)
        assert all(torch.equal(got, ilw.i8_linear(A, W, b, act=act, out_dtype=dtype)) for _ in range(2))
    ilw.device_status()


@pytest.mark.parametrize("M,N", [(1200, 2600), (1201, 2601), (333, 9000), (5001, 1026), (97, 20010)])
@pytest.mark.parametrize("K", [2200, 65])
def test_tiles_that_end_anywhere(ilw, M, N, K):
    """Columns and rows past the last tile, blocks of K that end in each half; results in rows that take wide stores and such that do not."""
    A, W = made(ilw, 1, M, K), made(ilw, 3, N, K, weights=True)
    for pad, dtype in ((0, torch.bfloat16), (3, torch.float16), (-N % 8, torch.float16)):
        wide = torch.full((M, N + pad + 8), 9.0, device="cuda", dtype=dtype)
        got = ilw.i8_linear(A, W, out=wide[:, :N])
        check_product(got, A, W, None, "none")
        got.fill_(9.0)
        assert bool((wide == 9).all())
    ilw.device_status()


@pytest.mark.parametrize("act,dtype", [("none", torch.float32), ("gelu", torch.bfloat16), ("silu_gate", torch.float16)])
@pytest.mark.parametrize("form,counts,N,K", [
    ("pair", [700, 0, 1, 333, 1024, 225, 95], 2304, 2600), ("pair", [700, 0, 1, 333, 1024, 225, 95], 1704, 600), ("few", [1, 0, 9], 300, 4200), ("few", [0, 2, 130, 0], 140, 8192),
    ("one", [5, 0, 1, 2] * 4, 1000, 700), ("one", [100] * 9, 514, 700), ("one", [40, 3, 0, 60], 2000, 1000), (4, [60, 0, 70], 520, 4200)])
def test_every_form_by_expert(ilw, form, counts, N, K, act, dtype):
    off, E = np.r_[0, np.cumsum(counts)], len(counts)
    M = int(off[-1])
    assert form_of(ilw, M, N, K, E, act, dtype)[0] == form
    A, W = made(ilw, 1, M, K), made(ilw, 3, E * N, K, weights=True)
    W = ilw.I8Tensor(W.codes.unflatten(0, (E, N)), W.scales.view(E, N))
    b = torch.randn((E, N), device="cuda", generator=generator(5))
    got = ilw.i8_grouped_linear(A, W, torch.from_numpy(off.astype(np.int32)).cuda(), b, act=act, out_dtype=dtype)
    for e in range(E):
        if counts[e]:
            s = slice(int(off[e]), int(off[e + 1]))
            check_product(got[s], ilw.I8Tensor(A.codes[s], A.scales[s]), ilw.I8Tensor(W.codes[e], W.scales[e]), b[e], act)
    ilw.device_status()


@pytest.mark.parametrize("form,M,N,K", [("one", 130, 1712, 500), (8, 40, 1000, 8200), (4, 130, 1000, 2100), (2, 16, 5000, 8200), ("pair", 5000, 2600, 500), ("pair", 3001, 514, 1030)])
def test_every_form_gives_up_a_bounded_wait(ilw, form, M, N, K):
    """A load that never comes (a debug hook skips one and shortens the waits): the kernel reports it and ends, and the next call is right."""
    assert form_of(ilw, M, N, K, None, "none", torch.bfloat16)[0] == form
    A, W = made(ilw, 1, M, K), made(ilw, 3, N, K, weights=True)
    want = ilw.i8_linear(A, W)
    assert ilw.lib().ilwdetr_debug_gemm_wait(0, 20_000_000) == 0
    try:
        ilw.i8_linear(A, W)
        with pytest.raises(ilw.IlwError, match="wait"):
            ilw.device_status()
    finally:
        assert ilw.lib().ilwdetr_debug_gemm_wait(-1, 0) == 0
    assert torch.equal(ilw.i8_linear(A, W), want)
    ilw.device_status()


def test_two_products_at_once(ilw):
    """Calls on two streams, each larger than half of the GPU, and a chain on each that reads what the call before it wrote."""
    A, W = made(ilw, 1, 3001, 1030), made(ilw, 3, 1712, 1030, weights=True)
    V = made(ilw, 7, 514, 1712, weights=True)
    want = ilw.i8_linear(ilw.i8_quantize(ilw.i8_linear(A, W, act="gelu")), V)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        with torch.cuda.stream(s):
            got += [ilw.i8_linear(ilw.i8_quantize(ilw.i8_linear(A, W, act="gelu")), V) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)
    ilw.device_status()


# ---------------------------------------------------------------------------- past 2^31 elements
def test_rows_past_32_bits(ilw):
    """The last rows of a matrix of more than 2^31 values are those that they are alone, there and back."""
    R, K = 270000, 8192
    x = torch.empty((R, K), dtype=torch.bfloat16, device="cuda").normal_(generator=generator(1))
    q = ilw.i8_quantize(x)
    last = ilw.i8_quantize(x[-300:])
    assert torch.equal(q.codes[-300:], last.codes) and torch.equal(q.scales[-300:], last.scales)
    at = torch.tensor([R - 1, 0, R - 2], dtype=torch.int32, device="cuda")
    some, want = ilw.i8_quantize(x, gather=at), ilw.i8_quantize(x[at.long()])
    assert torch.equal(some.codes, want.codes) and torch.equal(some.scales, want.scales)
    y = ilw.i8_dequantize(q, dtype=torch.bfloat16, out=x)
    assert torch.equal(y[-300:], ilw.i8_dequantize(last, dtype=torch.bfloat16))


@pytest.mark.parametrize("act", ["none", "silu_gate"])
def test_results_past_32_bits(ilw, act):
    """The last rows of a result of more than 2^31 values (sums below 2^24, so that the order of additions does not matter)."""
    M, N, K = 140000, 16400 * (2 if act == "silu_gate" else 1), 70
    A, W = ilw.i8_quantize(torch.randn((M, K), generator=generator(1), device="cuda")), made(ilw, 3, N, K, weights=True)
    y = ilw.i8_linear(A, W, act=act)
    for lo, hi in ((0, 130), (M - 130, M)):
        check_product(y[lo:hi], ilw.I8Tensor(A.codes[lo:hi], A.scales[lo:hi]), W, None, act)


@pytest.mark.parametrize("count", [1, 60])
def test_weights_past_32_bits(ilw, count):
    """The last of experts with more than 2^31 codes, by the kernel for few tokens and by tiles."""
    E, N, K = 36, 8200, 8192
    x = torch.empty((E * N, K), dtype=torch.bfloat16, device="cuda").normal_(generator=generator(1))
    q = ilw.i8_quantize(x)
    W = ilw.I8Tensor(q.codes.unflatten(0, (E, N)), q.scales.view(E, N))
    A = made(ilw, 3, E * count, K)
    offsets = torch.arange(0, E * count + 1, count, dtype=torch.int32, device="cuda")
    y = ilw.i8_grouped_linear(A, W, offsets, out_dtype=torch.float32)
    for e in (0, E - 2, E - 1):
        rows = slice(e * count, (e + 1) * count)
        check_product(y[rows], ilw.I8Tensor(A.codes[rows], A.scales[rows]), ilw.I8Tensor(W.codes[e], W.scales[e]), None, "none")


# ---------------------------------------------------------------------------- sums past 2^24
def of_codes(ilw, codes):
    m = ilw.i8_empty(*codes.shape)
    m.codes.copy_(codes)
    m.scales.fill_(1.0)
    return m


@pytest.mark.parametrize("lo", [0, -128])
@pytest.mark.parametrize("form,M,N,K", [("few", 3, 60, 9000), (8, 40, 1000, 8200), (4, 130, 1000, 2100), (2, 16, 5000, 8200), ("one", 130, 1712, 1100), ("pair", 3001, 1712, 1030), ("pair", 200, 1712, 2100),
                                        ("pair", 1500, 1000, 4200), ("pair", 1100, 5000, 32768), (8, 40, 1000, (1 << 17) - 1), ("pair", 600, 3000, (1 << 17) - 1)])
def test_fp32_results_have_exact_sums(ilw, form, M, N, K, lo):
    """Codes of one sign, and of both: the result is the whole number, rounded once, whatever form the call takes."""
    A, W = (of_codes(ilw, torch.randint(lo, 128, (n, K), generator=generator(n + K), device="cuda").to(torch.int8)) for n in (M, N))
    assert form_of(ilw, M, N, K, None, "none", torch.float32)[0] == form
    got = ilw.i8_linear(A, W, out_dtype=torch.float32)
    assert torch.equal(got, (A.codes.double() @ W.codes.double().T).float())
    assert torch.equal(got[:2], ilw.i8_linear(ilw.I8Tensor(A.codes[:2], A.scales[:2]), W, out_dtype=torch.float32))
    ilw.device_status()


@pytest.mark.parametrize("act", ["none", "gelu", "silu_gate"])
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("counts,N,K", [([700, 0, 1, 333, 1024, 225, 95], 1704, 2600), ([60, 0, 70], 520, 20000), ([5, 0, 1, 2] * 4, 1000, 1700)])
def test_long_sums_by_expert(ilw, counts, N, K, dtype, act):
    """Several tiles a CTA, each of several parts of K, scales and biases; sums held exactly where the results' type or K asks for it."""
    off, E = np.r_[0, np.cumsum(counts)], len(counts)
    A, W = (of_codes(ilw, torch.randint(-100, 128, (n, K), generator=generator(n + K), device="cuda").to(torch.int8)) for n in (int(off[-1]), E * N))
    A.scales.uniform_(1e-4, 1e-3, generator=generator(1))
    W.scales.uniform_(1e-4, 1e-3, generator=generator(2))
    b = torch.randn((E, N), device="cuda", generator=generator(5))
    got = ilw.i8_grouped_linear(A, ilw.I8Tensor(W.codes.unflatten(0, (E, N)), W.scales.view(E, N)), torch.from_numpy(off.astype(np.int32)).cuda(), b, act=act, out_dtype=dtype)
    for e in range(E):
        if counts[e]:
            s, w = slice(int(off[e]), int(off[e + 1])), slice(e * N, (e + 1) * N)
            check_product(got[s], ilw.I8Tensor(A.codes[s], A.scales[s]), ilw.I8Tensor(W.codes[w], W.scales[w]), b[e], act)
            if dtype == torch.float32 and act == "none":  # a sum rounded once, two factors and a bias
                z = A.codes[s].double() @ W.codes[w].double().T * A.scales[s].double()[:, None] * W.scales[w].double()
                assert bool(((got[s].double() - (z + b[e].double())).abs() <= 4 * 2.0**-24 * (2 * z.abs() + b[e].abs())).all())
    ilw.device_status()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("M", [1, 40, 400, 3000])
@pytest.mark.parametrize("K", [8192, 16384, 16385, (1 << 17) - 1])
def test_16_bit_results_of_long_sums(ilw, K, M, dtype):
    """Codes of one sign.  Up to K = 16384 a tile's sum loses less than a unit of 2^-23 with each 16 of K: 2^-13 in all, and half as much in norm; past that
    nothing.  The result then is off by that, by three roundings of fp32 and by its own."""
    A, W = (of_codes(ilw, torch.randint(0, 128, (n, K), generator=generator(n + K), device="cuda").to(torch.int8)) for n in (M, 1000))
    A.scales.fill_(2.0**-14)
    want = A.codes.double() @ W.codes.double().T * 2.0**-14
    got = ilw.i8_linear(A, W, out_dtype=dtype).double()
    off = K / 16 * 2.0**-23 if K <= 16384 else 0.0
    assert bool(((got - want).abs() <= (off + 3 * 2.0**-24 + EPS[dtype] * (1 + off)) * want).all())
    assert float((got - want).norm() / want.norm()) <= off / 2 + EPS[dtype]


# ---------------------------------------------------------------------------- scales
@pytest.mark.parametrize("form,M,N,K", [("few", 12, 40, 256), (4, 130, 1000, 2100), ("one", 130, 1712, 500), ("pair", 700, 1000, 1030)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_scales_of_every_size_meet(ilw, form, M, N, K, dtype):
    """Neither a large scale of a token nor one of a channel overflows, or a small one loses bits, where the result fits; a scale of 0
    leaves the bias."""
    assert form_of(ilw, M, N, K, None, "none", dtype)[0] == form
    A, W = (of_codes(ilw, torch.randint(-127, 128, (n, K), generator=generator(n), device="cuda").to(torch.int8)) for n in (M, N))
    sizes = torch.tensor([1.0, 1e36, 2.6e36, 1e30, 1e-30, 2.0**-126, 0.0, 1e10, 1e-10, 3.0])
    A.scales.copy_(sizes.repeat(M // 10 + 1)[:M])
    W.scales.copy_(sizes.repeat_interleave(4).repeat(N // 40 + 1)[:N])
    b = torch.randn(N, device="cuda", generator=generator(5))
    got = ilw.i8_linear(A, W, b, out_dtype=dtype)
    sums = A.codes.double() @ W.codes.double().T
    z = sums * A.scales.double()[:, None] * W.scales.double()
    want = z + b.double()
    # (a sum past 2^24 cannot be here; a product of two factors has two roundings, the bias one, the result one; below fp32's normal range they are of
    # its smallest step; whatever comes within those roundings of the largest number may round past it)
    lost = torch.where(sums.abs() >= 2.0**24, torch.inf, 0.0)
    assert not bool(lost.any())
    top = torch.finfo(dtype).max
    tol = 4 * 2.0**-24 * (2 * z.abs() + b.abs()) + EPS[dtype] * want.abs() + 1e-44
    inside, outside = want.abs() < top * (1 - 2.0**-7), want.abs() > top * (1 + 2.0**-7)
    assert bool(((got.double() - want).abs() <= tol)[inside].all())
    assert bool((got[outside] == torch.sign(want[outside]) * torch.inf).all()) and bool(outside.any()) and not bool(got.isnan().any())
    zero = A.scales == 0
    assert torch.equal(got[zero], b.to(dtype).expand(int(zero.sum()), N))
    assert torch.equal(got[:, W.scales == 0], b[W.scales == 0].to(dtype).expand(M, int((W.scales == 0).sum())))
    ilw.device_status()


@pytest.mark.parametrize("kind", ["MxExperts", "I8Experts"])
def test_experts_refuse_their_routing_at_once(ilw, kind):
    """What moe_route would refuse is refused with the weights, not in the first forward."""
    E, d, F = 8, 64, 96
    w1, w2 = torch.randn((E, 2 * F, d), generator=generator(1), device="cuda"), torch.randn((E, d, F), generator=generator(2), device="cuda")
    make = getattr(ilw, kind)
    for how in (dict(top=9), dict(top=2, bias=torch.zeros(7, device="cuda")), dict(top=2, bias=torch.zeros(8, dtype=torch.float16, device="cuda")), dict(top=2, groups=3),
                dict(top=2, score="tanh"), dict(top=5, groups=2, top_groups=1), dict(top=2, groups=4, top_groups=5), dict(top=2, scale=float("nan")),
                dict(top=2, groups=4, top_groups=2, group_best=3)):
        with pytest.raises(ilw.IlwError):
            make(w1, w2, **how)
    x, logits = torch.randn((50, d), generator=generator(3), device="cuda"), torch.randn((50, E), generator=generator(4), device="cuda")
    assert torch.equal(make(w1, w2, 2).forward(x, logits), make(w1, w2, 2, scale=1.0, groups=2, top_groups=2, score="softmax").forward(x, logits))


def test_offsets_at_the_ends_of_32_bits(ilw):
    """Whatever the offsets say, nothing outside the result is written, and ranges in order have their products."""
    A, W = made(ilw, 1, 600, 64), made(ilw, 3, 4 * 34, 64, weights=True)
    W = ilw.I8Tensor(W.codes.unflatten(0, (4, 34)), W.scales.view(4, 34))
    top, low = (1 << 31) - 1, -(1 << 31)
    for offsets in ([0, top, low, 600, 600], [low, low, top, top, top], [top, top, top, top, top], [low, 0, 300, 600, top], [low, top, low, top, low]):
        wide = torch.full((620, 34), 7.0, device="cuda")
        ilw.i8_grouped_linear(A, W, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=wide[10:610])
        assert bool((wide[:10] == 7).all()) and bool((wide[610:] == 7).all())
        if offsets == [low, 0, 300, 600, top]:
            for e in (1, 2):
                s = slice(300 * (e - 1), 300 * e)
                check_product(wide[10:610][s], ilw.I8Tensor(A.codes[s], A.scales[s]), ilw.I8Tensor(W.codes[e], W.scales[e]), None, "none")
    ilw.device_status()


def test_weights_past_32_bits_by_form(ilw):
    """The last of experts with more than 2^31 codes: by the kernel for few tokens, and by tiles."""
    E, N, K = 36, 8200, 8192
    x = torch.empty((E * N, K), dtype=torch.bfloat16, device="cuda").normal_(generator=generator(1))
    q = ilw.i8_quantize(x)
    del x
    W = ilw.I8Tensor(q.codes.unflatten(0, (E, N)), q.scales.view(E, N))
    for form, counts in (("few", {0: 1, E - 2: 1, E - 1: 2}), ("pair", {0: 9, 7: 30, E - 2: 70, E - 1: 33})):
        off = np.r_[0, np.cumsum([counts.get(e, 0) for e in range(E)])]
        M = int(off[-1])
        for dtype in (torch.float32, torch.bfloat16):
            assert form_of(ilw, M, N, K, E, "none", dtype)[0] == form
            A = made(ilw, 3, M, K)
            y = ilw.i8_grouped_linear(A, W, torch.from_numpy(off.astype(np.int32)).cuda(), out_dtype=dtype)
            for e in counts:
                s = slice(int(off[e]), int(off[e + 1]))
                check_product(y[s], ilw.I8Tensor(A.codes[s], A.scales[s]), ilw.I8Tensor(W.codes[e], W.scales[e]), None, "none")
    ilw.device_status()


@pytest.mark.parametrize("form,M,N,K,skipped", [("one", 130, 1712, 1100, 0), (8, 40, 1000, 8200, 0), (2, 16, 5000, 8200, 0), (2, 16, 5000, 8200, 9), ("pair", 3001, 1712, 2600, 0),
                                                ("pair", 3001, 1712, 2600, 9), ("pair", 3001, 1712, 2600, 30)])
def test_long_sums_give_up_a_bounded_wait(ilw, form, M, N, K, skipped):
    """As test_every_form_gives_up_a_bounded_wait, where sums are taken out of tensor memory on the way: a load of the first 1024 of K, of the next
    ones, of the second tile."""
    assert form_of(ilw, M, N, K, None, "none", torch.float32)[0] == form
    A, W = made(ilw, 1, M, K), made(ilw, 3, N, K, weights=True)
    want = ilw.i8_linear(A, W, out_dtype=torch.float32)
    assert ilw.lib().ilwdetr_debug_gemm_wait(skipped, 20_000_000) == 0
    try:
        ilw.i8_linear(A, W, out_dtype=torch.float32)
        with pytest.raises(ilw.IlwError, match="wait"):
            ilw.device_status()
    finally:
        assert ilw.lib().ilwdetr_debug_gemm_wait(-1, 0) == 0
    assert torch.equal(ilw.i8_linear(A, W, out_dtype=torch.float32), want)
    ilw.device_status()
