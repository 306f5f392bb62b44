"""Routing by scores, a bias and groups on the GPU against a plain restatement in 64 bits.

Experts, places and offsets are exact, ties included.  Weights: exponentials of at most 2 ulp whose arguments (differences of
logits) are off by half an ulp of at most 2^6 here, so 2^6 2^-24 relative; sums of at most E terms; and a few roundings."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def ilw():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import paper_2607_24981_gb300 as m
    from paper_2607_24981_gb300 import build

    build.build()
    m.lib()
    return m


def ref_route(x, k, renormalize, score="softmax", bias=None, groups=1, top_groups=None, group_best=2, scale=1.0):
    """float64 x [T, E] (numpy) -> expert, weight, offsets, source, slot."""
    T, E = x.shape
    # The scores of x and -x add up to 1 for every x: which of two such groups ranks better is a matter of the last bit of 64, so
    # that bit is taken where the operator says it takes it, from 1 / (1 + exp(-x)) on the device.
    sigmoids = (1 / (1 + torch.exp(-torch.from_numpy(x).cuda()))).cpu().numpy()
    x = np.where(np.isnan(x), -np.inf, x)
    expert, weight, size = np.full((T, k), -1), np.zeros((T, k)), E // groups
    for t in range(T):
        v = x[t]
        on = v > -np.inf
        if not on.any():
            continue
        with np.errstate(over="ignore", invalid="ignore"):
            p = np.where(on, np.where(v == v.max(), 1.0, np.exp(v - v.max())), 0)
            s = np.where(on, sigmoids[t], 0) if score == "sigmoid" else p / p.sum()
        c = s if bias is None else s + bias
        c = np.where(on & ~np.isnan(c), c, -np.inf)
        order = v if bias is None else c
        if groups > 1 and (top_groups or groups) < groups:
            rank = np.full(groups, -np.inf)
            for g in range(groups):
                of = (order if group_best == 1 else c)[g * size: (g + 1) * size]
                best = np.sort(of[of > -np.inf])[::-1][:group_best]
                if len(best):
                    rank[g] = best.sum()
            take = [g for g in np.argsort(-rank, kind="stable")[:top_groups] if rank[g] > -np.inf]
            order = np.where(np.isin(np.arange(E) // size, take), order, -np.inf)
        best = np.argsort(-order, kind="stable")[:k]
        best = best[order[best] > -np.inf]
        expert[t, : len(best)] = best
        if not len(best):
            continue
        if renormalize and score == "sigmoid":  # scores too small for 64 bits keep their ratios
            z = -np.logaddexp(0, -v[best])
            w = np.exp(z - z.max())
        else:
            w = s[best]
        weight[t, : len(best)] = scale * w / (w.sum() if renormalize else 1)
    entries = sorted((expert[t, j], t, j) for t in range(T) for j in range(k) if expert[t, j] >= 0)
    offsets = np.searchsorted([e for e, _, _ in entries], np.arange(E + 1))
    source, slot = np.full(T * k, -1), np.full((T, k), -1)
    for s, (_, t, j) in enumerate(entries):
        source[s], slot[t, j] = t, s
    return expert, weight, offsets, source, slot


def check(ilw, x, k, renormalize, bias=None, **how):
    """moe_route of x (a GPU tensor) against ref_route."""
    r = ilw.moe_route(x, k, renormalize, bias=bias, **how)
    expert, weight, offsets, source, slot = ref_route(x.double().cpu().numpy(), k, renormalize, bias=None if bias is None else bias.double().cpu().numpy(), **how)
    got = r.expert.cpu().numpy()
    assert np.array_equal(got, expert), f"{(got != expert).any(1).sum()} of {len(got)} tokens went elsewhere"
    for a, b in ((r.offsets, offsets), (r.source, source), (r.slot, slot)):
        assert np.array_equal(a.cpu().numpy(), b)
    err = np.abs(r.weight.double().cpu().numpy() - weight)
    assert (err <= (x.shape[1] + 64 + 16) * 2.0**-23 * np.abs(weight) + 1e-44).all(), (err / (np.abs(weight) + 1e-300)).max()
    return r


SHAPES = [(1, 1, 1, 1, 1), (1, 8, 2, 2, 1), (7, 33, 4, 3, 2), (33, 64, 8, 8, 4), (300, 130, 6, 10, 3), (17, 256, 8, 8, 4), (700, 512, 16, 32, 5), (3000, 16, 1, 4, 1), (9000, 6, 2, 3, 2),
          (260, 160, 6, 8, 3), (1500, 63, 6, 9, 3), (400, 128, 8, 1, 1), (257, 96, 4, 32, 16)]


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T,E,k,groups,top_groups", SHAPES)
def test_route_by_scores_matches_64_bits(ilw, T, E, k, groups, top_groups, dtype, score):
    """Many equal logits (a coarse grid), masked experts, whole groups and rows masked, NaN; with and without a bias."""
    rng = np.random.default_rng(T + E + k)
    x = np.round(rng.standard_normal((T, E)) * 4) / 4
    x[rng.random((T, E)) < 0.1] = -np.inf
    x[rng.random((T, E)) < 0.02] = np.nan
    x[rng.random(T) < 0.1] = -np.inf
    if groups > 1:
        x.reshape(T, groups, -1)[rng.random((T, groups)) < 0.2] = -np.inf
    wide = torch.from_numpy(np.pad(x, ((0, 0), (1, 2)))).to(dtype).cuda()
    x = wide[:, 1: 1 + E]
    bias = torch.from_numpy(0.1 * rng.standard_normal(E)).float().cuda()
    for b in (None, bias, torch.zeros_like(bias), torch.round(bias * 20) / 20):
        for best in (1, 2):
            check(ilw, x if best == 1 else x.contiguous(), k, b is None, bias=b, score=score, groups=groups, top_groups=top_groups, group_best=best, scale=2.5 if best == 1 else 1.0)
    ilw.device_status()


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("groups,top_groups,group_best", [(1, 1, 2), (8, 4, 2), (8, 3, 1)])
@pytest.mark.parametrize("T", [200, 4000])
def test_scores_that_32_bits_do_not_separate(ilw, T, groups, top_groups, group_best, score):
    """Biases that undo the scores' differences but for a few units of 2^-26 or none, so that fp32 scores tie or exchange their order."""
    rng = np.random.default_rng(T + groups)
    E = 64
    x = torch.from_numpy(rng.standard_normal(E)).float()
    s = torch.sigmoid(x.double()) if score == "sigmoid" else torch.softmax(x.double(), 0)
    bias = (0.75 - s).float().cuda()  # c = 0.75 but for the rounding of the bias, which differs from expert to expert
    rows = x.expand(T, E).clone()
    away = torch.from_numpy(rng.random((T, E)) < 0.3)
    rows = torch.where(away, float("-inf") if score == "sigmoid" else rows, rows).cuda()
    check(ilw, rows, 8, False, bias=bias, score=score, groups=groups, top_groups=top_groups, group_best=group_best)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("T,E,groups,top_groups,group_best", [(100, 256, 2, 1, 2), (60, 96, 32, 9, 2), (700, 256, 32, 9, 2), (300, 512, 4, 2, 1), (300, 112, 16, 7, 2), (1000, 24, 12, 5, 2)])
def test_groups_that_32_bits_do_not_separate(ilw, T, E, groups, top_groups, group_best, biased, score):
    """The groups of a token hold the same logits in another order, some of them one unit of fp32 larger."""
    rng, size = np.random.default_rng(T + E), E // groups
    same = rng.standard_normal((T, 1, size)).astype(np.float32)
    nudged = np.where(rng.random((T, groups, size)) < 0.3, np.nextafter(same, np.float32(np.inf)), same)
    x = rng.permuted(nudged, axis=2).reshape(T, E)
    x[rng.random((T, E)) < 0.02] = -np.inf
    bias = torch.full((E,), 0.125, device="cuda") if biased else None
    check(ilw, torch.from_numpy(x).cuda(), 3, True, bias=bias, score=score, groups=groups, top_groups=top_groups, group_best=group_best)


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 60, 64, 65, 111, 113, 224, 225, 256, 257, 511, 513])
def test_route_of_few_tokens(ilw, T):
    """Either side of where a CTA does all and of the lanes it gives a token; with 32 groups, ranks that leave no room for that."""
    rng = np.random.default_rng(T)
    for E, k, groups in ((8, 3, 2), (96, 5, 32), (112, 16, 14), (256, 5, 32)):
        x = np.round(rng.standard_normal((T, E)) * 4) / 4
        x[rng.random((T, E)) < 0.2] = -np.inf
        x = torch.from_numpy(x).float().cuda()
        bias = torch.from_numpy(0.1 * rng.standard_normal(E)).float().cuda()
        check(ilw, x, k, True, bias=bias, score="sigmoid", groups=groups, top_groups=max(groups // 2, 2))
        check(ilw, x, k, False, score="softmax", groups=groups, top_groups=max(groups // 2, 2), group_best=1)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E,k,groups,top_groups", [(128, 8, 8, 4), (256, 8, 1, 1), (63, 6, 9, 3)])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_many_random_tokens(ilw, score, E, k, groups, top_groups, dtype):
    """Enough tokens that some have neighbours that fp32 cannot tell apart; experts against plain operations in 64 bits on the GPU."""
    gen = torch.Generator("cuda").manual_seed(E + groups)
    x = (1.5 * torch.randn((60000, E), generator=gen, device="cuda")).to(dtype)
    bias = 0.1 * torch.randn(E, generator=gen, device="cuda")
    r = ilw.moe_route(x, k, score=score, bias=bias, groups=groups, top_groups=top_groups)
    c = (1 / (1 + torch.exp(-x.double())) if score == "sigmoid" else torch.softmax(x.double(), 1)) + bias.double()
    if groups > 1:
        of = c.view(-1, groups, E // groups)
        rank = torch.sort(of, dim=2, descending=True).values[..., :2].sum(2)
        stay = torch.zeros_like(rank, dtype=torch.bool).scatter_(1, torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :top_groups], True)
        c = torch.where(stay[..., None], of, -torch.inf).view(-1, E)
    assert torch.equal(r.expert.long(), torch.sort(c, dim=1, descending=True, stable=True).indices[:, :k])


def test_biases_that_pin_or_ban_experts(ilw):
    inf, nan = float("inf"), float("nan")
    bias = torch.tensor([0.0, 1e6, -1e6, -inf, nan, inf, 3e38, 0.0], device="cuda")
    x = torch.randn((50, 8), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    for score in ("sigmoid", "softmax"):
        r = check(ilw, x, 6, True, bias=bias, score=score)
        assert r.expert[:, :3].tolist() == [[5, 6, 1]] * 50 and r.expert[:, 5].tolist() == [2] * 50
        check(ilw, x, 3, True, bias=bias, score=score, groups=4, top_groups=2, group_best=2)
        check(ilw, x, 3, True, bias=bias, score=score, groups=4, top_groups=2, group_best=1)


def test_logits_of_every_size(ilw):
    """Infinities, the largest numbers, scores that are 1 or 0 in 64 bits, and weights of scores below fp32's range."""
    big, inf = float(np.float32(3.4028234e38)), float("inf")
    x = torch.tensor([[big, -big, 0.0, -0.0], [-big, -big, -big, -inf], [0.0, -0.0, -0.0, 0.0], [float("nan")] * 4, [inf, 1.0, 2.0, 3.0], [inf, inf, 0.0, -inf],
                      [-200.0, -201.0, -202.0, -300.0], [50.0, 60.0, 70.0, 55.0], [-90.0, -95.0, 0.0, -1.0], [-101.0, -100.0, -99.0, -98.0]]).cuda()
    zero = torch.zeros(4, device="cuda")
    for score in ("sigmoid", "softmax"):
        for bias in (None, zero, zero + 0.1):
            for renormalize in (True, False):
                check(ilw, x, 3, renormalize, score=score, bias=bias, scale=2.0)
                for best in (1, 2):
                    check(ilw, x, 2, renormalize, score=score, bias=bias, groups=2, top_groups=1, group_best=best)
    w = ilw.moe_route(x, 3, score="sigmoid").weight
    assert torch.allclose(w[6].cpu(), torch.softmax(torch.tensor([-200.0, -201.0, -202.0]), 0), rtol=1e-5)
    empty = ilw.moe_route(torch.empty((0, 6), device="cuda"), 2, score="sigmoid", groups=3, top_groups=2)
    assert empty.offsets.tolist() == [0] * 7 and empty.expert.shape == (0, 2)


@pytest.mark.parametrize("T,E,k,how", [(4000, 256, 8, dict(score="sigmoid")), (20000, 128, 4, dict(score="sigmoid", groups=8, top_groups=4)), (200, 64, 16, dict(score="softmax", scale=2.5)),
                                       (5000, 64, 6, dict(score="softmax", scale=2.5))])
@pytest.mark.parametrize("renormalize", [True, False])
def test_weights_as_exact_as_plain_operations(ilw, T, E, k, how, renormalize):
    """In norm, over many weights, no further from 64 bits than plain fp32 operations are (a tenth more for chance)."""
    x = 2 * torch.randn((T, E), device="cuda", generator=torch.Generator("cuda").manual_seed(T + E))
    r = ilw.moe_route(x, k, renormalize, **how)

    def weights(x):
        s = 1 / (1 + torch.exp(-x)) if how["score"] == "sigmoid" else torch.exp(x - x.amax(1, keepdim=True))
        s = s if how["score"] == "sigmoid" else s / s.sum(1, keepdim=True)
        top = torch.gather(s, 1, r.expert.long())
        return how.get("scale", 1.0) * (top / top.sum(1, keepdim=True) if renormalize else top)

    want = weights(x.double())
    assert (r.weight.double() - want).norm() <= 1.1 * (weights(x).double() - want).norm()


def test_defaults_are_those_of_plain_routing(ilw):
    """Without a bias, groups or a scale the scores' path gives what the plain one does."""
    x = torch.randn((3000, 64), generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    plain = ilw.moe_route(x, 4)
    same = ilw.moe_route(x, 4, groups=4, top_groups=4)
    for a, b in zip((plain.expert, plain.offsets, plain.source, plain.slot), (same.expert, same.offsets, same.source, same.slot)):
        assert torch.equal(a, b)
    assert torch.allclose(plain.weight, same.weight, rtol=2e-6, atol=0)


@pytest.mark.parametrize("T", [16, 2000])
def test_routing_follows_its_stream_and_graphs(ilw, T):
    x = [torch.randn((T, 64), generator=torch.Generator("cuda").manual_seed(i), device="cuda") for i in range(3)]
    how = dict(score="sigmoid", bias=torch.linspace(-0.1, 0.1, 64, device="cuda"), groups=8, top_groups=3)
    want = [ilw.moe_route(v, 4, **how) for v in x]
    graphs = []
    for i in range(2):
        b, g = x[0].clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = ilw.moe_route(b, 4, **how)
        graphs.append((b, g, r))
    for i, j in ((1, 2), (2, 0), (0, 1)):
        for (b, g, r), n in zip(graphs, (i, j)):
            b.copy_(x[n])
            g.replay()
        torch.cuda.synchronize()
        for (b, g, r), n in zip(graphs, (i, j)):
            assert all(torch.equal(u, v) for u, v in zip(r, want[n]))


def test_logits_past_32_bits(ilw):
    """The last tokens of more than 2^31 logits go where they go alone."""
    T, E = 8500000, 256
    x = torch.empty((T, E), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    how = dict(score="sigmoid", bias=torch.linspace(-0.1, 0.1, E, device="cuda"), groups=8, top_groups=4)
    r, alone = ilw.moe_route(x, 2, **how), ilw.moe_route(x[-500:], 2, **how)
    assert torch.equal(r.expert[-500:], alone.expert) and torch.equal(r.weight[-500:], alone.weight)
    assert torch.equal(torch.bincount(r.expert.flatten(), minlength=E).cumsum(0).int(), r.offsets[1:])
    assert torch.equal(r.source[r.slot[-500:].long()], torch.arange(T - 500, T, dtype=torch.int32, device="cuda")[:, None].expand(500, 2))


# Of a softmax that is renormalised only the taken logits count: their differences d from the largest of them are below 2^6 here and exact to
# 2^-24 d, the exponentials off by 2 ulp, and there are a sum of k terms, a quotient and a factor.
FAR = 2.0**6 * 2.0**-24 + (4 + 16 + 4) * 2.0**-23


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("T", [5, 300, 3000])
@pytest.mark.parametrize("groups,top_groups", [(1, 1), (8, 3)])
@pytest.mark.parametrize("away", [88.0, 104.0, 130.0, 3000.0, float("inf")])
def test_softmax_of_experts_far_below_the_largest(ilw, away, groups, top_groups, T, dtype):
    """Biases ban the experts with the largest logits (every other row: none of them has such); the weights of those taken are their softmax."""
    rng = np.random.default_rng(T + groups)
    E, k = 64, 6
    x = torch.from_numpy(4 * rng.standard_normal((T, E))).to(dtype)
    ban = torch.arange(E) % 5 == 3
    x[::2, ban] += away
    bias = torch.where(ban, torch.tensor([-1e6, -float("inf")])[torch.arange(E) % 2], torch.from_numpy(0.3 * rng.permutation(E)).float())
    x, bias = x.cuda(), bias.cuda()
    r = ilw.moe_route(x, k, True, score="softmax", bias=bias, groups=groups, top_groups=top_groups, scale=1.5)
    assert not bool(ban.cuda()[r.expert.long()].any())
    want = 1.5 * torch.softmax(torch.gather(x.double(), 1, r.expert.long()), 1)
    assert bool(((r.weight.double() - want).abs() <= FAR * want + 1e-44).all())
    if away < float("inf"):  # (the restatement takes a softmax of the row)
        expert = ref_route(x.double().cpu().numpy(), k, False, "softmax", bias.double().cpu().numpy(), groups, top_groups)[0]
        assert np.array_equal(r.expert.cpu().numpy(), expert)


def test_a_taken_infinity_takes_all_the_weight(ilw):
    """Among taken logits +inf is the limit of large ones; several share."""
    inf = float("inf")
    x = torch.tensor([[inf, 0.0, 1.0, 2.0], [inf, inf, 0.0, 1.0], [0.0, -150.0, -151.0, inf], [-200.0, 0.0, -200.0, -201.0]]).cuda()
    bias = torch.tensor([0.0, 0.0, 0.0, -1e6]).cuda()
    w = ilw.moe_route(x, 3, True, score="softmax", bias=bias).weight
    assert w[0].tolist() == [1.0, 0.0, 0.0] and w[1].tolist() == [0.5, 0.5, 0.0] and w[2].tolist() == [1.0, 0.0, 0.0]
    one = ilw.moe_route(torch.tensor([[0.0, -120.0]]).cuda(), 1, True, score="softmax", bias=torch.tensor([0.0, 10.0]).cuda())
    assert one.expert.tolist() == [[1]] and one.weight.tolist() == [[1.0]]


def check_groups(ilw, x, bias, k, **how):
    """The experts of moe_route of x (a GPU tensor) are those of ref_route."""
    got = ilw.moe_route(x, k, False, bias=bias, **how).expert.cpu().numpy()
    want = ref_route(x.double().cpu().numpy(), k, False, bias=bias.double().cpu().numpy(), **how)[0]
    assert np.array_equal(got, want), f"{(got != want).any(1).sum()} of {len(got)} tokens went elsewhere"


def test_a_group_of_large_biases_between_two_others(ilw):
    """Ranks in 64 bits: 1.24267, 1.34267, 1.24266, 1.24265, of which the first is off by some 10^-4 in fp32 and the others by 10^-6."""
    def logits(rank):  # of two equal scores that add up to rank
        return [float(np.log(rank / 2 / (1 - rank / 2)))] * 2

    x = torch.tensor([logits(1.24267) + logits(1.34267) + logits(1.24266) + logits(1.24265)] * 40, device="cuda")
    for B in (100.0, 1e3, 1e4, 1e6):
        for at in range(4):  # the group of both signs
            bias = torch.zeros(8, device="cuda")
            bias[2 * at], bias[2 * at + 1] = B, -B
            for top_groups in (1, 2, 3):
                check_groups(ilw, x, bias, 2, score="sigmoid", groups=4, top_groups=top_groups, group_best=2)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("B", [1e3, 1e6])
@pytest.mark.parametrize("T,E,groups,top_groups", [(200, 64, 16, 6), (30000, 6, 3, 1), (20000, 16, 8, 3), (20000, 64, 32, 9)])
def test_large_biases_that_cancel_within_groups(ilw, T, E, groups, top_groups, B, score):
    """Some groups have biases +B and -B, so ranks that are off by hundreds of times what their neighbours' are."""
    rng, size = np.random.default_rng(T + E), E // groups
    bias = np.zeros(E, np.float32)
    for g in range(0, groups, 3):
        bias[g * size], bias[(g + 1) * size - 1] = B, -B
        bias[g * size + 1: (g + 1) * size - 1] = -2 * B
    x = rng.standard_normal((T, E)).astype(np.float32) * 0.3
    check_groups(ilw, torch.from_numpy(x).cuda(), torch.from_numpy(bias).cuda(), 2, score=score, groups=groups, top_groups=top_groups, group_best=2)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("T", [7, 400])
def test_ranks_past_the_largest_fp32_number(ilw, T, sign):
    """Sums of two biases that 64 bits hold and 32 do not; which are the larger is told, and a group of them is one."""
    bias = sign * torch.tensor([3e38, 2e38, 3e38, 2.5e38, 3.1e38, 2.2e38, 1.5e38, 3.2e38], device="cuda")
    x = torch.randn((T, 8), generator=torch.Generator("cuda").manual_seed(T), device="cuda")
    x[T // 2:, 2] = -float("inf")
    for top_groups in (1, 2, 3):
        check_groups(ilw, x, bias, 2, score="sigmoid", groups=4, top_groups=top_groups, group_best=2)
        check_groups(ilw, x, bias, 2, score="softmax", groups=4, top_groups=top_groups, group_best=1)
