"""Cases of the feed-forward operators: the root-mean-square norm with an 8-bit output, the gated
activation with an 8-bit output, the product with 4-bit weights and group scales, the routing of tokens
to experts, and the products of the experts that they are routed to.

Every operator is here in its plain form (32-bit torch operations, rounded once at the end), in 64 bits
(``exact``), and, with ``own`` set, as the calls of this package that a user makes.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
MIN_SCALE = 2.0 ** -64       # smallest scale of an 8-bit row: a row of zeros is zeros with this scale
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f16": 2, "f32": 4, "e4m3": 1}


def listed():
    return [
        # one token's row: latency counts
        {"name": "norm 1x4096 bf16", "op": "norm", "m": 1, "k": 4096, "type": "bf16", "residual": True, "pad": 0},
        # a prompt of odd length and width, rows of a wider buffer, the residual stream updated on the way
        {"name": "norm 4099x12345 f16", "op": "norm", "m": 4099, "k": 12345, "type": "f16", "residual": True, "pad": 7},
        # the gate and up halves of one product's output: a small batch in generation at an odd width, and a prompt
        {"name": "gate 33x2047 f16", "op": "gate", "m": 33, "f": 2047, "type": "f16"},
        {"name": "gate 4096x16384 bf16", "op": "gate", "m": 4096, "f": 16384, "type": "bf16"},
        # one token against a square matrix: the smallest call of generation
        {"name": "w4 1x4096x4096 e4m3", "op": "w4", "m": 1, "n": 4096, "k": 4096, "group": 128, "zeros": False, "type": "e4m3", "out": "bf16", "pad": 0},
        # a few requests at odd sizes: the last group, the last rows and the last pair of nibbles are cut short
        {"name": "w4 7x4099x12345 f16", "op": "w4", "m": 7, "n": 4099, "k": 12345, "group": 64, "zeros": True, "type": "f16", "out": "f16", "pad": 3},
        # a batch in generation, the down projection of a block
        {"name": "w4 48x4096x16384 bf16", "op": "w4", "m": 48, "n": 4096, "k": 16384, "group": 32, "zeros": False, "type": "bf16", "out": "bf16", "pad": 0},
        # a long prompt with the 8-bit rows that the norm gives
        {"name": "w4 4096x16384x4096 e4m3", "op": "w4", "m": 4096, "n": 16384, "k": 4096, "group": 128, "zeros": True, "type": "e4m3", "out": "bf16", "pad": 0},
        # one token among 256 experts in 8 groups of which 4 count, sigmoid scores with a bias for balance
        {"name": "route 1x256 sigmoid", "op": "route", "m": 1, "e": 256, "top": 8, "score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4, "type": "f32"},
        # a prompt among 64 experts, softmax scores
        {"name": "route 16384x64 softmax", "op": "route", "m": 16384, "e": 64, "top": 8, "score": "softmax", "bias": False, "groups": 1, "top_groups": 1, "type": "bf16"},
        # one token, its 8 experts of 64, the weighted sum of their outputs
        {"name": "experts 1 of 64x2048x2048", "op": "experts", "m": 1, "e": 64, "top": 8, "n": 2048, "k": 2048, "group": 128, "zeros": False, "type": "bf16",
         "out": "bf16", "each": True, "weighted": True},
        # a prompt's first product: the rows that the norm gives, one output row for each of a token's experts
        {"name": "experts 2048 of 64x2048x2048", "op": "experts", "m": 2048, "e": 64, "top": 8, "n": 2048, "k": 2048, "group": 128, "zeros": False, "type": "e4m3",
         "out": "bf16", "each": False, "weighted": False},
    ]


def _size(rng, lo, hi):
    """A size from lo to hi, spread over its logarithm; one in two is a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and hi >= 64:
        v = max(64, (v + 32) // 64 * 64)
    return max(lo, min(hi, v))


def _rows(rng, hi):
    return max(1, min(hi, int(round(math.exp(rng.uniform(0.0, math.log(hi)))))))


def _product(rng, case, most):
    """Sizes of the weights, types and groups, for at most ``most`` weights."""
    n, k = _size(rng, 64, most), _size(rng, 64, most)
    case.update(n=n, k=k, group=rng.choice([32, 64, 128]), zeros=rng.random() < 0.5, type=rng.choice(["bf16", "f16", "e4m3"]))
    case["out"] = case["type"] if case["type"] != "e4m3" else rng.choice(["bf16", "f16"])
    return case


def draw(rng):
    op = rng.choice(["norm", "gate", "w4", "w4", "route", "experts"])
    if op == "norm":
        return {"op": op, "m": _rows(rng, 4096), "k": _size(rng, 64, 16384), "type": rng.choice(["bf16", "f16", "f32"]),
                "residual": rng.random() < 0.7, "pad": rng.choice([0, 0, 8, 5])}
    if op == "gate":
        return {"op": op, "m": _rows(rng, 4096), "f": _size(rng, 64, 16384), "type": rng.choice(["bf16", "f16", "f32"])}
    if op == "w4":
        case = _product(rng, {"op": op, "m": _rows(rng, 4096), "pad": rng.choice([0, 0, 16, 3])}, 16384)
        case["m"] = max(1, min(case["m"], 4096 * 16384 * 4096 // (case["n"] * case["k"])))
        return case
    if op == "route":
        sigmoid = rng.random() < 0.5
        groups = rng.choice([1, 2, 4, 8])
        e = groups * _size(rng, 4, 512 // groups)
        top_groups = rng.randint(1, groups)
        return {"op": op, "m": _rows(rng, 16384), "e": e, "top": rng.randint(1, min(16, e // groups * top_groups)), "score": "sigmoid" if sigmoid else "softmax",
                "bias": sigmoid, "groups": groups, "top_groups": top_groups, "type": rng.choice(["bf16", "f16", "f32"])}
    e = _size(rng, 4, 128)
    case = _product(rng, {"op": op, "m": _rows(rng, 2048), "e": e, "top": rng.randint(1, min(8, e)), "each": rng.random() < 0.5, "weighted": rng.random() < 0.5}, 4096)
    while case["e"] * case["n"] * case["k"] > 64 * 2048 * 2048:
        case["e"] = max(1, case["e"] // 2)
        case["top"] = min(case["top"], case["e"])
        case["n"] = min(case["n"], 64 * 2048 * 2048 // (case["e"] * case["k"]))
    return case


def work(case):
    m, op = case["m"], case["op"]
    t = SIZE[case["type"]]
    if op == "norm":
        mk = m * case["k"]
        res = 2 if case["residual"] else 0       # the residual is read and the sum is written
        return {"bytes": mk * t * (1 + res) + case["k"] * t + mk + 4 * m, "flops": 6 * mk}
    if op == "gate":
        mf = m * case["f"]
        return {"bytes": 2 * mf * t + mf + 4 * m, "flops": 6 * mf}
    if op == "route":
        return {"bytes": m * case["e"] * t + (4 * case["e"] if case["bias"] else 0) + 8 * m * case["top"], "flops": 4 * m * case["e"]}
    n, k = case["n"], case["k"]
    groups = -(-k // case["group"])
    weights = n * -(-k // 2) + 2 * n * groups + (-(-n * groups // 2) if case["zeros"] else 0)
    scale = 4 if case["type"] == "e4m3" else 0
    if op == "w4":
        return {"bytes": weights + m * (k * t + scale) + m * n * SIZE[case["out"]], "flops": 2 * m * n * k}
    pairs = m * case["top"]
    used = case["e"] * (1 - (1 - case["top"] / case["e"]) ** m)      # experts that some token is expected to choose
    rows_in, rows_out = pairs if case["each"] else m, m if case["weighted"] else pairs
    return {"bytes": used * weights + rows_in * (k * t + scale) + rows_out * n * SIZE[case["out"]] + pairs * (8 if case["weighted"] else 4), "flops": 2 * pairs * n * k}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _stream(g, m, k, pad, dtype):
    """Rows as a model's residual stream has them: normal, a scale for each row, a few columns with larger values."""
    v = torch.randn(m, k + pad, device="cuda", generator=g)
    v *= torch.rand(m, 1, device="cuda", generator=g) * 2 + 0.25
    v *= 1 + 7 * (torch.rand(k + pad, device="cuda", generator=g) < 0.004)
    return v.to(dtype)[:, :k]


def _inputs(case, seed):
    g, m, dtype = _generator(seed), case["m"], TYPES[case["type"]]
    if case["op"] == "norm":
        s = {"x": _stream(g, m, case["k"], case["pad"], dtype)}
        s["r"] = _stream(g, m, case["k"], case["pad"], dtype) if case["residual"] else None
        s["w"] = (1 + 0.2 * torch.randn(case["k"], device="cuda", generator=g)).to(dtype)
        return s
    if case["op"] == "gate":
        return {"gu": _stream(g, m, 2 * case["f"], 0, dtype)}
    if case["op"] == "route":
        # a router's logits: some experts are liked more than others
        logits = torch.randn(m, case["e"], device="cuda", generator=g) * 1.5 + 0.5 * torch.randn(case["e"], device="cuda", generator=g)
        return {"logits": logits.to(dtype), "bias": 0.1 * torch.randn(case["e"], device="cuda", generator=g) if case["bias"] else None}
    n, k, group = case["n"], case["k"], case["group"]
    s, rows = {"xs": None}, m
    if case["op"] == "experts":
        likes = 0.5 * torch.randn(case["e"], device="cuda", generator=g)
        score, ids = (torch.randn(m, case["e"], device="cuda", generator=g) + likes).topk(case["top"], 1)
        s["ids"], s["weights"] = ids.to(torch.int32), torch.softmax(score, 1) if case["weighted"] else None
        n, rows = case["e"] * n, m * case["top"] if case["each"] else m
    groups = -(-k // group)
    v = torch.zeros(n, groups * group, device="cuda")
    v[:, :k] = torch.randn(n, k, device="cuda", generator=g) * 0.02
    v = v.view(n, groups, group)
    if case["zeros"]:
        lo, hi = v.amin(-1).clamp_max(0.0), v.amax(-1).clamp_min(0.0)
        scale = ((hi - lo) / 15).clamp_min(1e-6)
        zero = (-lo / scale).round().clamp(0, 15)
    else:
        scale = (v.abs().amax(-1) / 7).clamp_min(1e-6)
        zero = torch.full_like(scale, 8.0)
    q = ((v / scale[..., None]).round() + zero[..., None]).clamp(0, 15).to(torch.uint8).view(n, groups * group)[:, :k]
    if k % 2:
        q = torch.cat([q, torch.zeros(n, 1, dtype=torch.uint8, device="cuda")], 1)
    s["q"], s["s"] = (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous(), scale.to(TYPES[case["out"]])
    s["z"] = zero.to(torch.uint8) if case["zeros"] else None
    if case["op"] == "experts":
        s.update({name: s[name].view(case["e"], case["n"], -1) for name in ("q", "s", "z") if s[name] is not None})
    pad = case.get("pad", 0)
    if case["type"] == "e4m3":
        x = _stream(g, rows, k, pad, torch.float32)
        s["xs"] = x.abs().amax(-1).clamp_min(1e-6) / E4M3_MAX
        s["x"] = (torch.nn.functional.pad(x, (0, pad)) / s["xs"][:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(dtype)[:, :k]
    else:
        s["x"] = _stream(g, rows, k, pad, dtype)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_1202_3173_b200 as sw
        m = case["m"]
        # the buffers and the laid-out weights that a serving program keeps
        if case["op"] == "norm":
            s["out"] = sw.quant_rows(m, case["k"], "cuda") + ((torch.empty_like(s["r"]),) if case["residual"] else ())
        elif case["op"] == "gate":
            s["out"] = sw.quant_rows(m, case["f"], "cuda")
        elif case["op"] == "route":
            s["out"] = (torch.empty(m, case["top"], dtype=torch.int32, device="cuda"), torch.empty(m, case["top"], device="cuda"))
        elif case["op"] == "w4":
            s["matrix"] = sw.W4Matrix(s["q"], s["s"], s["z"], k=case["k"], group=case["group"])
            s["out"] = torch.empty(m, case["n"], dtype=TYPES[case["out"]], device="cuda")
        else:
            s["matrix"] = sw.W4Experts(s["q"], s["s"], s["z"], k=case["k"], group=case["group"])
            s["out"] = torch.empty(m if case["weighted"] else m * case["top"], case["n"], dtype=TYPES[case["out"]], device="cuda")
    return s


# ---- one pass --------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        import paper_1202_3173_b200 as sw
        if case["op"] == "norm":
            return sw.rms_norm_quant(state["x"], state["w"], EPS, residual=state["r"], out=state["out"])
        if case["op"] == "gate":
            f = case["f"]
            return sw.silu_mul_quant(state["gu"][:, :f], state["gu"][:, f:], out=state["out"])
        if case["op"] == "route":
            return sw.route_experts(state["logits"], case["top"], score=case["score"], bias=state["bias"], groups=case["groups"],
                                    top_groups=case["top_groups"], renormalize=True, out=state["out"])
        if case["op"] == "experts":
            return state["matrix"](state["x"], state["ids"], state["xs"], weights=state["weights"], out=state["out"])
        return state["matrix"](state["x"], state["xs"], out=state["out"])
    return {"norm": _norm, "gate": _gate, "w4": _w4, "route": _route, "experts": _experts}[case["op"]](state, case)


def _rows_to_8_bits(v):
    s = (v.abs().amax(-1) / E4M3_MAX).clamp_min(MIN_SCALE)
    return (v / s[:, None]).to(torch.float8_e4m3fn), s


def _norm(state, case):
    h = state["x"].float()
    if case["residual"]:
        h = h + state["r"].float()
    inv = (h * h).mean(-1, keepdim=True).add(EPS).rsqrt()
    q, s = _rows_to_8_bits(h * inv * state["w"].float())
    return (q, s, h.to(TYPES[case["type"]])) if case["residual"] else (q, s)


def _gate(state, case):
    f = case["f"]
    g, u = state["gu"][:, :f].float(), state["gu"][:, f:].float()
    return _rows_to_8_bits(g / (1 + (-g).exp()) * u)


def _weights(q, scale, zero, k, group):
    """The matrix (or matrices) in 32 bits."""
    q = torch.stack([q & 15, q >> 4], -1).flatten(-2)[..., :k].float()
    zero = zero.float().repeat_interleave(group, -1)[..., :k] if zero is not None else 8.0
    return scale.float().repeat_interleave(group, -1)[..., :k] * (q - zero)


def _w4(state, case):
    y = state["x"].float() @ _weights(state["q"], state["s"], state["z"], case["k"], case["group"]).t()
    if state["xs"] is not None:
        y = y * state["xs"][:, None]
    return y.to(TYPES[case["out"]])


def _route(state, case):
    logits = state["logits"].float()
    m, e, groups = case["m"], case["e"], case["groups"]
    if case["score"] == "softmax":
        score = (logits - logits.amax(1, keepdim=True)).exp()
        score = score / score.sum(1, keepdim=True)
        key = logits                                  # the same order as the scores'
    else:
        score = 1 / (1 + (-logits).exp())
        key = score + state["bias"] if case["bias"] else score
    if groups > 1:
        best = key.view(m, groups, -1).sort(dim=-1, descending=True).values
        best = best[..., 0] if case["score"] == "softmax" else best[..., 0] + best[..., 1]
        chosen = best.sort(dim=1, descending=True, stable=True).indices[:, :case["top_groups"]]
        left_out = torch.ones(m, groups, dtype=torch.bool, device="cuda").scatter_(1, chosen, False)
        key = key.masked_fill(left_out.repeat_interleave(e // groups, 1), -math.inf)
    ids = key.sort(dim=1, descending=True, stable=True).indices[:, :case["top"]]
    weights = score.gather(1, ids)
    return ids.to(torch.int32), weights / weights.sum(1, keepdim=True)


def _experts(state, case):
    m, e, top, k, group = case["m"], case["e"], case["top"], case["k"], case["group"]
    ids = state["ids"].flatten().long()
    x = state["x"].float()
    if state["xs"] is not None:
        x = x * state["xs"][:, None]
    if not case["each"]:
        x = x.repeat_interleave(top, 0)
    q, s, z = state["q"], state["s"], state["z"]
    if m * top <= e:                                  # few rows: each with its own expert's matrix
        w = _weights(q[ids], s[ids], z[ids] if z is not None else None, k, group)
        y = (w @ x[:, :, None])[..., 0]
    else:                                             # rows sorted by expert, as many for each as the fullest has
        order = ids.argsort(stable=True)
        count = torch.bincount(ids, minlength=e)
        place = torch.arange(m * top, device="cuda") - (count.cumsum(0) - count)[ids[order]]
        room = torch.zeros(e, int(count.max()), k, device="cuda")
        room[ids[order], place] = x[order]
        y = torch.empty(m * top, case["n"], device="cuda")
        y[order] = (room @ _weights(q, s, z, k, group).transpose(1, 2))[ids[order], place]
    if case["weighted"]:
        y = (y.view(m, top, -1) * state["weights"][..., None]).sum(1)
    return y.to(TYPES[case["out"]])


# ---- the same in 64 bits -----------------------------------------------------------------------------------------

def _product64(x, q, s, z, case):
    """Group by group: y = sum_g (x_g . (Q_g - Z_g) S_g)."""
    d, k, group = torch.float64, case["k"], case["group"]
    y = torch.zeros(x.shape[0], case["n"], dtype=d, device="cuda")
    nibbles = torch.empty(case["n"], 2 * q.shape[1], dtype=d, device="cuda")
    nibbles[:, 0::2] = (q % 16).to(d)
    nibbles[:, 1::2] = (q // 16).to(d)
    for i in range(-(-k // group)):
        a, b = i * group, min(k, (i + 1) * group)
        zero = 8.0 if z is None else z[:, i].to(d)[:, None]
        y.addmm_(x[:, a:b], ((nibbles[:, a:b] - zero) * s[:, i].to(d)[:, None]).t())
    return y


def exact(case, seed):
    s = _inputs(case, seed)
    d = torch.float64
    if case["op"] == "norm":
        total = s["x"].to(d) if s["r"] is None else s["x"].to(d) + s["r"].to(d)
        values = total / torch.sqrt(torch.einsum("mk,mk->m", total, total) / case["k"] + EPS)[:, None] * s["w"].to(d)
    elif case["op"] == "gate":
        gate, up = s["gu"].to(d).split(case["f"], 1)
        values = gate * torch.special.expit(gate) * up
    elif case["op"] == "route":
        # the ids are whole numbers and have no value here; the weights of the experts that the definition chooses, in order
        score = torch.softmax(s["logits"].to(d), 1) if case["score"] == "softmax" else torch.special.expit(s["logits"].to(d))
        key = score + s["bias"].to(d) if case["bias"] else score
        size = case["e"] // case["groups"]
        if case["groups"] > 1:
            two = key.unflatten(1, (case["groups"], size)).topk(min(size, 1 if case["score"] == "softmax" else 2), 2).values.sum(2)
            keep = torch.zeros_like(two).scatter_(1, two.topk(case["top_groups"], 1).indices, 1.0).repeat_interleave(size, 1)
            key = torch.where(keep > 0, key, torch.full_like(key, -9.0))
        chosen = torch.gather(score, 1, key.topk(case["top"], 1).indices)
        return None, chosen / chosen.sum(1, keepdim=True)
    elif case["op"] == "experts":
        # expert by expert, over the tokens that chose it
        factor = torch.ones(case["m"], case["top"], dtype=d, device="cuda") if s["weights"] is None else s["weights"].to(d)
        y = torch.zeros(case["m"], case["top"], case["n"], dtype=d, device="cuda")
        x = s["x"].to(d) if s["xs"] is None else s["x"].to(d) * s["xs"].to(d)[:, None]
        for i in range(case["e"]):
            token, slot = torch.nonzero(s["ids"] == i, as_tuple=True)
            if token.numel():
                rows = x[token * case["top"] + slot] if case["each"] else x[token]
                y[token, slot] = _product64(rows, s["q"][i], s["s"][i], None if s["z"] is None else s["z"][i], case) * factor[token, slot][:, None]
        return y.sum(1) if case["weighted"] else y.flatten(0, 1)
    else:
        y = _product64(s["x"].to(d), s["q"], s["s"], s["z"], case)
        return y if s["xs"] is None else y * s["xs"].to(d)[:, None]
    scale = torch.maximum(values.abs().max(1).values / E4M3_MAX, torch.full((case["m"],), MIN_SCALE, dtype=d, device="cuda"))
    out = (values / scale[:, None], scale)
    return out + (total,) if case["op"] == "norm" and s["r"] is not None else out
