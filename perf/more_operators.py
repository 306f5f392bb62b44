"""Performance cases of the 8-bit integer products with float scales and of the routing by scores, biases and groups.

Every case is one operator: quantising rows to int8 with a scale each (and reading the values back), the product of such rows,
the product grouped by expert, and routing to experts with a bias for balance and groups of experts.  ``run`` computes it in
plain torch operations, or, with ``own`` set, through the package's entry points.  ``exact`` restates each operator in 64 bits.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}
_TINY = 2.0**-126  # the least scale of a row that is not all zeros


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # the hidden rows of a Medium feed-forward at 8 images of 1600 tokens, quantised for its second product
        {"name": "quantize_hidden", "op": "quantize", "rows": 12800, "k": 1536, "type": "bf16", "gather": 0},
        # fp32 tokens of an odd width, each gathered for its two experts and quantised on the way
        {"name": "quantize_gather", "op": "quantize", "rows": 1201, "k": 2051, "type": "f32", "gather": 2},
        # one token of a serving loop against a square layer: the weights' bytes and latency
        {"name": "linear_one_token", "op": "linear", "m": 1, "n": 4096, "k": 4096, "act": "none", "bias": False, "type": "bf16"},
        # the decoder's 300 queries through a layer of odd sizes, fp32 results
        {"name": "linear_queries", "op": "linear", "m": 300, "n": 1001, "k": 1030, "act": "none", "bias": True, "type": "f32"},
        # the first product of a Medium feed-forward at 8 images, with its GELU: a short K, the epilogue counts
        {"name": "linear_fc1_gelu", "op": "linear", "m": 12800, "n": 1536, "k": 384, "act": "gelu", "bias": True, "type": "bf16"},
        # a long batch through a wide layer: the tensor cores' rate
        {"name": "linear_large", "op": "linear", "m": 8192, "n": 8192, "k": 8192, "act": "none", "bias": False, "type": "bf16"},
        # 16 tokens of a serving step, two experts each of 64: the weights of the experts met, few rows each
        {"name": "grouped_decode", "op": "grouped", "rows": 32, "experts": 64, "n": 4096, "k": 2048, "act": "silu_gate",
         "bias": False, "type": "bf16", "skew": 0.5},
        # a prompt of 8192 tokens, two experts each of 32, gated
        {"name": "grouped_prompt", "op": "grouped", "rows": 16384, "experts": 32, "n": 8192, "k": 2048, "act": "silu_gate",
         "bias": False, "type": "bf16", "skew": 0.3},
        # the decoder's 300 queries of 16 images, two experts each of 13 of odd widths, some of them empty, fp32 results
        {"name": "grouped_queries", "op": "grouped", "rows": 9600, "experts": 13, "n": 1001, "k": 250, "act": "none",
         "bias": True, "type": "f32", "skew": 1.5},
        # routing of a serving step: 16 tokens, 256 experts in 8 groups of which 4 are taken
        {"name": "route_decode", "op": "route", "tokens": 16, "experts": 256, "top": 8, "type": "f32", "score": "sigmoid", "bias": True,
         "groups": 8, "top_groups": 4, "group_best": 2, "masked": 0.0, "renormalize": True, "scale": 2.5},
        # routing of long prompts, some experts masked per row and some rows masked whole
        {"name": "route_long", "op": "route", "tokens": 65536, "experts": 128, "top": 8, "type": "bf16", "score": "sigmoid", "bias": True,
         "groups": 8, "top_groups": 4, "group_best": 2, "masked": 0.1, "renormalize": True, "scale": 1.0},
        # the decoder's queries of 16 images by softmax, limited to 3 of 9 groups by the best expert of each
        {"name": "route_queries", "op": "route", "tokens": 4800, "experts": 63, "top": 6, "type": "f16", "score": "softmax", "bias": False,
         "groups": 9, "top_groups": 3, "group_best": 1, "masked": 0.0, "renormalize": False, "scale": 16.0},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "grouped", "grouped", "route", "route"])
    kind = rng.choice(["bf16", "f16", "f32"])
    if op == "quantize":
        k = _log(rng, 17, 8192)
        gather = rng.choice([0, 0, 1, 2, 4])
        return {"op": op, "rows": _log(rng, 1, max(1, min(32768, (1 << 25) // (k * max(1, gather))))), "k": k, "type": kind, "gather": gather}
    if op == "linear":
        n, k = 2 * _log(rng, 8, 4096), _log(rng, 33, 8192)
        act = rng.choice(["none", "gelu", "silu_gate"])
        m = _log(rng, 1, max(1, min(32768, int(1.5e11 / (n * k)))))
        return {"op": op, "m": m, "n": n - (act != "silu_gate" and rng.random() < 0.3), "k": k, "act": act, "bias": rng.random() < 0.5, "type": kind}
    if op == "grouped":
        experts, n, k = _log(rng, 2, 128), 2 * _log(rng, 32, 2048), _log(rng, 33, 4096)
        n = max(2, min(n, 2 * ((1 << 29) // (2 * experts * k))))
        act = rng.choice(["none", "gelu", "silu_gate"])
        rows = _log(rng, 1, max(1, min(32768, int(1e11 / (n * k)))))
        return {"op": op, "rows": rows, "experts": experts, "n": n - (act != "silu_gate" and n > 2 and rng.random() < 0.3), "k": k, "act": act,
                "bias": rng.random() < 0.5, "type": kind, "skew": round(rng.uniform(0.0, 1.0), 2)}
    groups = rng.choice([1, 1, 2, 4, 8, rng.randint(2, 16)])
    experts = groups * _log(rng, max(1, 4 // groups), 256 // groups)
    top_groups = rng.randint(1, groups)
    return {"op": op, "tokens": _log(rng, 1, 65536), "experts": experts, "top": rng.randint(1, min(8, experts // groups * top_groups)), "type": kind,
            "score": rng.choice(["sigmoid", "softmax"]), "bias": rng.random() < 0.6, "groups": groups, "top_groups": top_groups,
            "group_best": rng.choice([1, 2]), "masked": rng.choice([0.0, 0.0, 0.1, 0.5]), "renormalize": rng.random() < 0.5,
            "scale": rng.choice([1.0, 2.5])}


def _counts(case):
    """Rows of each expert: the case's rows dealt out with weights (rank + 1)^-skew, the ranks in a shuffled order."""
    rng = random.Random(case["rows"] * 1009 + case["experts"])
    weights = [(i + 1) ** -case["skew"] for i in range(case["experts"])]
    rng.shuffle(weights)
    got = [0] * case["experts"]
    for e in rng.choices(range(case["experts"]), weights, k=case["rows"]):
        got[e] += 1
    return got


def work(case):
    op, size = case["op"], _SIZE[case["type"]]
    if op == "quantize":
        out = case["rows"] * max(1, case["gather"])
        return {"bytes": (case["rows"] + out) * case["k"] * size, "flops": 0}
    if op in ("linear", "grouped"):
        n, k = case["n"], case["k"]
        rows = case["m"] if op == "linear" else case["rows"]
        met = 1 if op == "linear" else sum(c > 0 for c in _counts(case))  # the experts that have rows
        wide = n // 2 if case["act"] == "silu_gate" else n
        return {"bytes": (rows + met * n) * (k + 4) + rows * wide * size + (4 * met * n if case["bias"] else 0), "flops": 2.0 * rows * n * k}
    t, e, k = case["tokens"], case["experts"], case["top"]
    return {"bytes": t * e * size + t * k * 16 + 4 * (e + 1) + (4 * e if case["bias"] else 0), "flops": 0}


# ---------------------------------------------------------------------------- inputs
def _encode(x):
    """Codes (as float64) and scales of the rows of x [..., K] in int8: a row's scale is its largest magnitude over 127, in
    fp32, and its codes are its values over the scale, to the nearest and of two the even one."""
    amax = x.float().abs().amax(-1)
    fine = torch.isfinite(amax)
    scale = torch.where(fine, torch.where(amax > 0, (amax / 127.0).clamp(min=_TINY), 0.0), math.nan)
    code = torch.round(x.double() / scale.double().unsqueeze(-1)).clamp(-127, 127)
    return torch.where((fine & (amax > 0)).unsqueeze(-1), code, 0.0), scale


def _packed(x):
    """x [..., K] as int8 codes, rows of which start on 16-byte boundaries, and scales."""
    code, scale = _encode(x)
    k = x.shape[-1]
    codes = torch.zeros(*x.shape[:-1], -(-k // 16) * 16, dtype=torch.int8, device=x.device)
    codes[..., :k] = code
    return codes[..., :k], scale


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def _activations(gen, rows, k):
    """Rows as a normalisation leaves them: a few channels are much larger than the rest, and some rows are padding."""
    x = _normal(gen, rows, k) * torch.exp(0.7 * _normal(gen, k))
    return x * (torch.rand(rows, 1, generator=gen, device="cuda") >= 0.02) if rows > 8 else x


def _weights(gen, *shape):
    return _normal(gen, *shape) / math.sqrt(shape[-1])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, dt = case["op"], _DT[case["type"]]
    s = dict(case)
    if op == "quantize":
        s["x"] = _activations(gen, case["rows"], case["k"]).to(dt)
        if case["gather"]:
            at = torch.arange(case["rows"], device="cuda").repeat_interleave(case["gather"])
            s["at"] = at[torch.randperm(at.numel(), generator=gen, device="cuda")].int()
    elif op in ("linear", "grouped"):
        rows = case["m"] if op == "linear" else case["rows"]
        s["a"] = _packed(_activations(gen, rows, case["k"]))
        if op == "linear":
            s["w"] = _packed(_weights(gen, case["n"], case["k"]))
            s["b"] = 0.1 * _normal(gen, case["n"]) if case["bias"] else None
        else:
            counts, e, n, k = _counts(case), case["experts"], case["n"], case["k"]
            codes = torch.zeros(e, n, -(-k // 16) * 16, dtype=torch.int8, device="cuda")[..., :k]
            scales = torch.empty(e, n, device="cuda")
            for i in range(e):
                codes[i], scales[i] = _packed(_weights(gen, n, k))
            s["w"] = codes, scales
            s["b"] = 0.1 * _normal(gen, e, n) if case["bias"] else None
            s["offsets"] = torch.tensor([sum(counts[:i]) for i in range(e + 1)], dtype=torch.int32, device="cuda")
            s["most"] = max(counts)
    else:
        x = 1.5 * _normal(gen, case["tokens"], case["experts"])
        if case["masked"]:
            off = torch.rand(x.shape, generator=gen, device="cuda") < case["masked"]
            off |= torch.rand(case["tokens"], 1, generator=gen, device="cuda") < 0.1 * case["masked"]
            x = x.masked_fill(off, -math.inf)
        s["x"] = x.to(dt)
        s["b"] = 0.1 * _normal(gen, case["experts"]) if case["bias"] else None
    return s


# ---------------------------------------------------------------------------- the operators
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2607_24981_gb300 as ilw

    op, dt = s["op"], _DT[s["type"]]
    if op == "quantize":
        return ilw.i8_dequantize(ilw.i8_quantize(s["x"], gather=s.get("at")), dt)
    if op == "linear":
        return ilw.i8_linear(ilw.I8Tensor(*s["a"]), ilw.I8Tensor(*s["w"]), bias=s["b"], act=s["act"], out_dtype=dt)
    if op == "grouped":
        return ilw.i8_grouped_linear(ilw.I8Tensor(*s["a"]), ilw.I8Tensor(*s["w"]), s["offsets"], bias=s["b"], act=s["act"], out_dtype=dt)
    r = ilw.moe_route(s["x"], s["top"], renormalize=s["renormalize"], score=s["score"], bias=s["b"], groups=s["groups"],
                      top_groups=s["top_groups"], group_best=s["group_best"], scale=s["scale"])
    return {"expert": r.expert, "weight": r.weight, "offsets": r.offsets, "source": r.source, "slot": r.slot}


def _activate(z, act):
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu_gate":
        gate, up = z[..., 0::2], z[..., 1::2]
        return gate / (1.0 + torch.exp(-gate)) * up
    return z


def _run_plain(s):
    op, dt = s["op"], _DT[s["type"]]
    if op == "quantize":
        x = s["x"] if s.get("at") is None else s["x"][s["at"].long()]
        code, scale = _encode(x)
        return (code.float() * scale.unsqueeze(-1)).to(dt)
    if op == "linear":
        (a, sa), (w, sw) = s["a"], s["w"]
        z = a.float() @ w.float().T * sa[:, None] * sw
        return _activate(z if s["b"] is None else z + s["b"], s["act"]).to(dt)
    if op == "grouped":
        (a, sa), (w, sw), off = s["a"], s["w"], s["offsets"].long()
        at = (off[:-1, None] + torch.arange(s["most"], device=a.device)).clamp(max=a.shape[0] - 1)
        z = torch.bmm(a[at].float(), w.float().mT) * sa[at][..., None] * sw[:, None]
        z = _activate(z if s["b"] is None else z + s["b"][:, None], s["act"]).to(dt)
        row = torch.arange(a.shape[0], device=a.device)
        expert = (row[:, None] >= off[None, 1:]).sum(1)
        return z[expert, row - off[expert]]
    return _route(s)


def _scores(x, score):
    """Scores of logits that are -inf where an expert is never taken."""
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-x))
    p = torch.exp(x - x.amax(1, keepdim=True).clamp(min=-3e38))
    return p / p.sum(1, keepdim=True).clamp(min=1.0)


def _route(s):
    x, k, bias, groups = s["x"].float(), s["top"], s["b"], s["groups"]
    t, e = x.shape
    x = torch.where(x > -math.inf, x, -math.inf)
    # who is taken, in 64 bits: two experts may lie closer to each other than a rounding of 32 bits
    value = _scores(x.double(), s["score"]) + (0.0 if bias is None else bias.double())
    value = torch.where(x > -math.inf, value, -math.inf)
    choice = x.double() if bias is None else value  # (without a bias: the order of the logits)
    if groups > 1:
        of = (choice if s["group_best"] == 1 else value).view(t, groups, -1)
        best = torch.sort(of, dim=2, descending=True).values[..., : s["group_best"]]
        rank = torch.where(best > -math.inf, best, 0.0).sum(2)
        rank = torch.where(best[..., 0] > -math.inf, rank, -math.inf)
        taken = torch.zeros(t, groups, dtype=torch.bool, device=x.device)
        taken.scatter_(1, torch.sort(rank, dim=1, descending=True, stable=True).indices[:, : s["top_groups"]], True)
        choice = torch.where(taken[..., None], choice.view(t, groups, -1), -math.inf).view(t, e)
    top, expert = torch.sort(choice, dim=1, descending=True, stable=True)
    expert, taken = expert[:, :k], top[:, :k] > -math.inf
    weight = torch.where(taken, _scores(x, s["score"]).gather(1, expert), 0.0)
    if s["renormalize"]:
        weight = torch.where(taken, weight / weight.sum(1, keepdim=True), 0.0)
    weight = weight * s["scale"]
    flat = torch.where(taken, expert, e).flatten()
    order = torch.argsort(flat, stable=True)
    offsets = (flat[None, :] < torch.arange(e + 1, device=x.device)[:, None]).sum(1)
    place = torch.empty_like(order)
    place[order] = torch.arange(t * k, device=x.device)
    return {"expert": torch.where(taken, expert, -1).int(), "weight": weight, "offsets": offsets.int(),
            "source": torch.where(flat[order] < e, order // k, -1).int(), "slot": torch.where(taken, place.view(t, k), -1).int()}


# ---------------------------------------------------------------------------- 64 bits
def _finish64(z, act):
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if act == "silu_gate":
        return torch.sigmoid(z[:, 0::2]) * z[:, 0::2] * z[:, 1::2]
    return z


def _weights64(s):
    """Routing weights: the experts taken one after the other, each the first of the largest that are left."""
    x = s["x"].double()
    t, e = x.shape
    on = x > -math.inf
    whole = torch.logsumexp(torch.where(on, x, -math.inf), 1, keepdim=True)
    log_score = torch.nn.functional.logsigmoid(x) if s["score"] == "sigmoid" else x - whole
    log_score = torch.where(on, log_score, -math.inf)
    value = torch.exp(log_score) if s["b"] is None else torch.exp(log_score) + s["b"].double()
    value = torch.where(on, value, -math.inf)
    left = torch.where(on, x, -math.inf) if s["b"] is None else value.clone()
    if s["groups"] > 1:
        size, ranks = e // s["groups"], []
        for g in range(s["groups"]):
            if s["group_best"] == 1:
                ranks.append(left[:, g * size: (g + 1) * size].max(1).values)
            else:
                part = value[:, g * size: (g + 1) * size]
                two = torch.topk(part, min(2, size), dim=1).values
                ranks.append(torch.where(torch.isinf(two[:, 0]), -math.inf, torch.where(torch.isinf(two), 0.0, two).sum(1)))
        rank, taken = torch.stack(ranks, 1), torch.zeros(t, s["groups"], dtype=torch.bool, device=x.device)
        for _ in range(s["top_groups"]):
            at = (rank == rank.max(1, keepdim=True).values).double().argmax(1, keepdim=True)
            taken.scatter_(1, at, True)
            rank = rank.scatter(1, at, -math.inf)
        left = torch.where(taken.repeat_interleave(size, 1), left, -math.inf)
    chosen = torch.full((t, s["top"]), -math.inf, dtype=torch.float64, device=x.device)
    for j in range(s["top"]):
        best = left.max(1, keepdim=True).values
        at = (left == best).double().argmax(1, keepdim=True)
        chosen[:, j: j + 1] = torch.where(best > -math.inf, log_score.gather(1, at), -math.inf)
        left.scatter_(1, at, -math.inf)
    if s["renormalize"]:
        chosen = chosen - torch.logsumexp(chosen, 1, keepdim=True)
    return s["scale"] * torch.exp(chosen).nan_to_num(nan=0.0)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        x = s["x"].double() if s.get("at") is None else s["x"].double()[s["at"].long()]
        largest = torch.maximum(x.max(1).values, -x.min(1).values)
        scale = (largest / 127).float().double().clamp(min=_TINY)  # (as it is held)
        units = x / scale[:, None]
        below = torch.floor(units)
        up = (units - below > 0.5) | ((units - below == 0.5) & (torch.remainder(below, 2) == 1))
        return (below + up) * scale[:, None]
    if op == "linear":
        a, w = (c.double() * v.double()[:, None] for c, v in (s["a"], s["w"]))
        z = a @ w.T
        return _finish64(z if s["b"] is None else z + s["b"].double(), case["act"])
    if op == "grouped":
        a, off, parts = s["a"][0].double() * s["a"][1].double()[:, None], s["offsets"].tolist(), []
        for e in range(case["experts"]):
            z = a[off[e]: off[e + 1]] @ (s["w"][0][e].double() * s["w"][1][e].double()[:, None]).T
            parts.append(_finish64(z if s["b"] is None else z + s["b"][e].double(), case["act"]))
        return torch.cat(parts)
    return {"expert": None, "weight": _weights64(s), "offsets": None, "source": None, "slot": None}
