"""Performance cases of the microscaled 4-bit and mixture-of-experts operators.

Every case is one operator: quantising rows to MXFP4 (and reading the values back), the MXFP4 product, the product grouped by
expert, routing and combination.  ``run`` computes it in plain 32-bit torch operations, or, with ``own`` set, through the
package's entry points.  ``exact`` restates each operator in 64 bits.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_SIZE = {"bf16": 2, "f16": 2, "f32": 4}


# ---------------------------------------------------------------------------- cases
def listed():
    return [
        # the hidden rows of a Medium feed-forward at 8 images of 1600 tokens, quantised for its second product
        {"name": "quantize_hidden", "op": "quantize", "rows": 12800, "k": 1536, "type": "bf16", "gather": 0},
        # fp32 tokens of an odd width, each gathered for its two experts and quantised on the way
        {"name": "quantize_gather", "op": "quantize", "rows": 1201, "k": 2051, "type": "f32", "gather": 2},
        # one token of a serving loop against a square layer: the weights' bytes and latency
        {"name": "linear_one_token", "op": "linear", "m": 1, "n": 4096, "k": 4096, "act": "none", "bias": False, "type": "bf16"},
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
        # routing of a serving step
        {"name": "route_decode", "op": "route", "tokens": 16, "experts": 64, "top": 4, "type": "bf16", "masked": 0.0, "renormalize": True},
        # routing of long prompts, some experts masked per row and some rows masked whole
        {"name": "route_long", "op": "route", "tokens": 65536, "experts": 128, "top": 8, "type": "f32", "masked": 0.1, "renormalize": False},
        # the decoder's queries joined from two experts onto their residual, fp32
        {"name": "combine_queries", "op": "combine", "tokens": 4800, "top": 2, "n": 256, "type": "f32", "residual": True, "dropped": 0.05},
        # a long batch joined from eight experts
        {"name": "combine_long", "op": "combine", "tokens": 16384, "top": 8, "n": 4096, "type": "bf16", "residual": False, "dropped": 0.0},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "grouped", "grouped", "route", "combine"])
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
    if op == "route":
        experts = _log(rng, 4, 256)
        return {"op": op, "tokens": _log(rng, 1, 65536), "experts": experts, "top": rng.randint(1, min(8, experts)), "type": kind,
                "masked": rng.choice([0.0, 0.0, 0.1, 0.5]), "renormalize": rng.random() < 0.5}
    n, top = _log(rng, 33, 8192), rng.randint(1, 8)
    return {"op": "combine", "tokens": _log(rng, 1, max(1, min(65536, (1 << 26) // (n * top)))), "top": top, "n": n, "type": kind,
            "residual": rng.random() < 0.5, "dropped": rng.choice([0.0, 0.1])}


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
        return {"bytes": case["rows"] * case["k"] * size + out * case["k"] * 2, "flops": 0}
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        wide = n // 2 if case["act"] == "silu_gate" else n
        return {"bytes": (m + n) * k * 17 / 32 + m * wide * size + (4 * n if case["bias"] else 0), "flops": 2.0 * m * n * k}
    if op == "grouped":
        r, n, k = case["rows"], case["n"], case["k"]
        met = sum(c > 0 for c in _counts(case))
        wide = n // 2 if case["act"] == "silu_gate" else n
        return {"bytes": (r + met * n) * k * 17 / 32 + r * wide * size + (4 * met * n if case["bias"] else 0), "flops": 2.0 * r * n * k}
    if op == "route":
        t, e, k = case["tokens"], case["experts"], case["top"]
        return {"bytes": t * e * size + t * k * 16 + 4 * (e + 1), "flops": 0}
    t, k, n = case["tokens"], case["top"], case["n"]
    return {"bytes": t * k * (n * size + 8) + t * n * size * (2 if case["residual"] else 1), "flops": 2.0 * t * k * n}


# ---------------------------------------------------------------------------- inputs
def _scales(dev):
    """The 256 E8M0 scales 2^(b - 127) and their inverses (255 stands for NaN)."""
    b = torch.arange(256, dtype=torch.float64, device=dev) - 127.0
    s, r = torch.exp2(b), torch.exp2(-b)
    s[255] = r[255] = float("nan")
    return s.float(), r.float()


def _levels(dev):
    """The 16 E2M1 values by code."""
    v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=dev)
    return torch.cat([v, -v])


def _blocks(x):
    """x [..., K] as zero-filled blocks of 32."""
    k = x.shape[-1]
    return torch.nn.functional.pad(x, (0, -k % 32)).unflatten(-1, (-1, 32))


def _encode(x):
    """Codes [..., blocks, 32] and scale bytes [..., blocks] of x in MXFP4."""
    v = _blocks(x.float())
    amax = v.abs().amax(-1)
    fine = torch.isfinite(amax)
    byte = (torch.frexp(torch.where(fine, amax, 1.0))[1].long() - 3).clamp(-127, 127) + 127
    byte = torch.where(amax == 0, 0, torch.where(fine, byte, 255))
    y = v * _scales(x.device)[1][byte].unsqueeze(-1)
    mag = y.abs()
    code = ((mag > 0.25).long() + (mag >= 0.75) + (mag > 1.25) + (mag >= 1.75) + (mag > 2.5) + (mag >= 3.5) + (mag > 5.0))
    return code + 8 * (y < 0), byte


def _packed(x):
    """x [..., K] as the two arrays of an MXFP4 tensor: codes two to a byte, the lower nibble first, rows of 16 ceil(K / 32)
    bytes; scale bytes in rows of a multiple of 16."""
    code, byte = _encode(x)
    code = code.flatten(-2)
    codes = (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8)
    scales = torch.nn.functional.pad(byte, (0, -byte.shape[-1] % 16)).to(torch.uint8)
    return codes.contiguous(), scales.contiguous()


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
            counts, e, n = _counts(case), case["experts"], case["n"]
            parts = [_packed(_weights(gen, n, case["k"])) for _ in range(e)]
            s["w"] = tuple(torch.stack([p[i] for p in parts]) for i in (0, 1))
            s["b"] = 0.1 * _normal(gen, e, n) if case["bias"] else None
            s["offsets"] = torch.tensor([sum(counts[:i]) for i in range(e + 1)], dtype=torch.int32, device="cuda")
            s["most"] = max(counts)
    elif op == "route":
        x = 2.0 * _normal(gen, case["tokens"], case["experts"])
        if case["masked"]:
            off = torch.rand(x.shape, generator=gen, device="cuda") < case["masked"]
            off |= torch.rand(case["tokens"], 1, generator=gen, device="cuda") < 0.1 * case["masked"]
            x = x.masked_fill(off, float("-inf"))
        s["x"] = x.to(dt)
    else:
        t, k = case["tokens"], case["top"]
        s["y"] = _normal(gen, t * k, case["n"]).to(dt)
        s["slot"] = torch.randperm(t * k, generator=gen, device="cuda").int().view(t, k)
        s["slot"] = s["slot"].masked_fill(torch.rand(t, k, generator=gen, device="cuda") < case["dropped"], -1)
        s["weight"] = torch.softmax(_normal(gen, t, k), 1)
        s["residual"] = _normal(gen, t, case["n"]).to(dt) if case["residual"] else None
    return s


# ---------------------------------------------------------------------------- the operators
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    import paper_2607_24981_gb300 as ilw

    op, dt = s["op"], _DT[s["type"]]
    if op == "quantize":
        return ilw.mx_dequantize(ilw.mx_quantize(s["x"], gather=s.get("at")), torch.bfloat16)
    if op == "linear":
        return ilw.mx_linear(ilw.MxTensor(*s["a"], s["k"]), ilw.MxTensor(*s["w"], s["k"]), bias=s["b"], act=s["act"], out_dtype=dt)
    if op == "grouped":
        return ilw.mx_grouped_linear(ilw.MxTensor(*s["a"], s["k"]), ilw.MxTensor(*s["w"], s["k"]), s["offsets"], bias=s["b"],
                                     act=s["act"], out_dtype=dt)
    if op == "route":
        r = ilw.moe_route(s["x"], s["top"], renormalize=s["renormalize"])
        return {"expert": r.expert, "weight": r.weight, "offsets": r.offsets, "source": r.source, "slot": r.slot}
    return ilw.moe_combine(s["y"], s["slot"], s["weight"], residual=s["residual"])


def _values(packed, k):
    """The fp32 values of an MXFP4 tensor."""
    codes, scales = packed
    level, scale = _levels(codes.device), _scales(codes.device)[0]
    v = torch.stack([level[(codes & 15).long()], level[(codes >> 4).long()]], -1).flatten(-2).unflatten(-1, (-1, 32))
    return (v * scale[scales.long()[..., : v.shape[-2]]].unsqueeze(-1)).flatten(-2)[..., :k]


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
        code, byte = _encode(x)
        v = _levels(x.device)[code] * _scales(x.device)[0][byte].unsqueeze(-1)
        return v.flatten(-2)[..., : s["k"]].to(torch.bfloat16)
    if op == "linear":
        z = _values(s["a"], s["k"]) @ _values(s["w"], s["k"]).T
        return _activate(z if s["b"] is None else z + s["b"], s["act"]).to(dt)
    if op == "grouped":
        a, off = _values(s["a"], s["k"]), s["offsets"].long()
        at = off[:-1, None] + torch.arange(s["most"], device=a.device)
        z = torch.bmm(a[at.clamp(max=a.shape[0] - 1)], _values(s["w"], s["k"]).mT)
        z = _activate(z if s["b"] is None else z + s["b"][:, None], s["act"]).to(dt)
        row = torch.arange(a.shape[0], device=a.device)
        expert = (row[:, None] >= off[None, 1:]).sum(1)
        return z[expert, row - off[expert]]
    if op == "route":
        return _route(s["x"].float(), s["top"], s["renormalize"])
    y = s["y"].float()[s["slot"].long().clamp(min=0)] * s["weight"][..., None]
    out = torch.where(s["slot"][..., None] >= 0, y, 0.0).sum(1)
    return (out if s["residual"] is None else out + s["residual"].float()).to(dt)


def _route(x, k, renormalize):
    t, e = x.shape
    x = torch.where(x > float("-inf"), x, float("-inf"))
    top, expert = torch.sort(x, dim=1, descending=True, stable=True)
    p = torch.exp(x - top[:, :1])
    top, expert = top[:, :k], expert[:, :k]
    taken = top > float("-inf")
    q = torch.where(taken, torch.exp(top - top[:, :1]), 0.0)
    weight = torch.where(taken, q / (q.sum(1, keepdim=True) if renormalize else p.sum(1, keepdim=True)), 0.0)
    flat = torch.where(taken, expert, e).flatten()
    order = torch.argsort(flat, stable=True)
    offsets = (flat[None, :] < torch.arange(e + 1, device=x.device)[:, None]).sum(1)
    rank = torch.empty_like(order)
    rank[order] = torch.arange(t * k, device=x.device)
    return {"expert": torch.where(taken, expert, -1).int(), "weight": weight, "offsets": offsets.int(),
            "source": torch.where(flat[order] < e, order // k, -1).int(), "slot": torch.where(taken, rank.view(t, k), -1).int()}


# ---------------------------------------------------------------------------- 64 bits
def _decode64(packed, k):
    """An MXFP4 tensor in float64, from the bits of its codes: sign, two exponent bits, one mantissa bit."""
    codes, scales = (t.long() for t in packed)
    nibble = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=torch.long, device=codes.device)
    nibble[..., 0::2], nibble[..., 1::2] = codes % 16, codes // 16
    exponent, mantissa = (nibble // 2) % 4, (nibble % 2).double()
    v = torch.where(exponent > 0, torch.exp2(exponent.double() - 1) * (1 + mantissa / 2), mantissa / 2)
    v = torch.where(nibble >= 8, -v, v)
    return v[..., :k] * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)[..., :k]


def _finish64(z, act):
    if act == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if act == "silu_gate":
        return torch.sigmoid(z[:, 0::2]) * z[:, 0::2] * z[:, 1::2]
    return z


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "quantize":
        x = s["x"].double()
        x = x if s.get("at") is None else x[s["at"].long()]
        v = torch.zeros(x.shape[0], -(-case["k"] // 32) * 32, dtype=torch.float64, device=x.device)
        v[:, : case["k"]] = x
        v = v.view(x.shape[0], -1, 32)
        amax = v.abs().amax(2, keepdim=True)
        exponent = (amax.view(torch.int64) >> 52) - 1023  # floor(log2 amax), from the bits of the double
        scale = torch.ldexp(torch.ones_like(amax), exponent.clamp(-125, 129) - 2)
        grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
        best, dist = torch.zeros_like(v), torch.full_like(v, math.inf)
        for i in (0, 2, 4, 6, 1, 3, 5, 7):  # the even codes first: a tie stays with them
            d = ((v / scale).abs() - grid[i]).abs()
            best, dist = torch.where(d < dist, grid[i], best), torch.minimum(d, dist)
        return (torch.sign(v) * best * scale).nan_to_num(nan=0.0).view(x.shape[0], -1)[:, : case["k"]]
    if op == "linear":
        z = _decode64(s["a"], case["k"]) @ _decode64(s["w"], case["k"]).T
        return _finish64(z if s["b"] is None else z + s["b"].double(), case["act"])
    if op == "grouped":
        a, off, parts = _decode64(s["a"], case["k"]), s["offsets"].tolist(), []
        for e in range(case["experts"]):
            z = a[off[e]: off[e + 1]] @ _decode64((s["w"][0][e], s["w"][1][e]), case["k"]).T
            parts.append(_finish64(z if s["b"] is None else z + s["b"][e].double(), case["act"]))
        return torch.cat(parts)
    if op == "route":
        x = s["x"].double()
        top = torch.full((case["tokens"], case["top"]), -math.inf, dtype=torch.float64, device=x.device)
        left = x.clone()
        for j in range(case["top"]):
            best = left.max(1).values
            at = (left == best[:, None]).double().argmax(1, keepdim=True)
            top[:, j] = best
            left.scatter_(1, at, -math.inf)
        whole = torch.logsumexp(top if case["renormalize"] else x, 1, keepdim=True)
        return {"expert": None, "weight": torch.exp(top - whole).nan_to_num(nan=0.0), "offsets": None, "source": None, "slot": None}
    out = torch.zeros(case["tokens"], case["n"], dtype=torch.float64, device="cuda")
    for j in range(case["top"]):
        on = s["slot"][:, j] >= 0
        out[on] += s["weight"][on, j, None].double() * s["y"][s["slot"][on, j].long()].double()
    return out if s["residual"] is None else out + s["residual"].double()
