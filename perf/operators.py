"""Cases of the feed-forward operators: the root-mean-square norm with an 8-bit output, the gated
activation with an 8-bit output, and the product with 4-bit weights and group scales.

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
        # one token's row at the widths of a small and of a wide model: latency counts
        {"name": "norm 1x4096 bf16", "op": "norm", "m": 1, "k": 4096, "type": "bf16", "residual": True, "pad": 0},
        # a batch of requests in generation, odd width, rows of a wider buffer
        {"name": "norm 37x12345 f16", "op": "norm", "m": 37, "k": 12345, "type": "f16", "residual": True, "pad": 7},
        # a long prompt, the residual stream updated on the way
        {"name": "norm 16384x4096 bf16", "op": "norm", "m": 16384, "k": 4096, "type": "bf16", "residual": True, "pad": 0},
        # the gate and up halves of one product's output: one token, a small odd batch, a prompt
        {"name": "gate 1x16384 bf16", "op": "gate", "m": 1, "f": 16384, "type": "bf16"},
        {"name": "gate 33x2047 f16", "op": "gate", "m": 33, "f": 2047, "type": "f16"},
        {"name": "gate 4096x16384 bf16", "op": "gate", "m": 4096, "f": 16384, "type": "bf16"},
        # one token against a square matrix: the smallest call of generation
        {"name": "w4 1x4096x4096 e4m3", "op": "w4", "m": 1, "n": 4096, "k": 4096, "group": 128, "zeros": False, "type": "e4m3", "out": "bf16", "pad": 0},
        # one token against a wide matrix with zero points, 16-bit activations
        {"name": "w4 1x16384x4096 bf16", "op": "w4", "m": 1, "n": 16384, "k": 4096, "group": 128, "zeros": True, "type": "bf16", "out": "bf16", "pad": 0},
        # a few requests at odd sizes: the last group, the last rows and the last pair of nibbles are cut short
        {"name": "w4 7x4099x12345 f16", "op": "w4", "m": 7, "n": 4099, "k": 12345, "group": 64, "zeros": True, "type": "f16", "out": "f16", "pad": 3},
        # a batch in generation, the down projection of a block
        {"name": "w4 48x4096x16384 bf16", "op": "w4", "m": 48, "n": 4096, "k": 16384, "group": 32, "zeros": False, "type": "bf16", "out": "bf16", "pad": 0},
        # a short prompt with the 8-bit rows that the norm gives
        {"name": "w4 512x16384x4096 e4m3", "op": "w4", "m": 512, "n": 16384, "k": 4096, "group": 128, "zeros": True, "type": "e4m3", "out": "bf16", "pad": 0},
        # a long prompt
        {"name": "w4 4096x16384x4096 bf16", "op": "w4", "m": 4096, "n": 16384, "k": 4096, "group": 128, "zeros": False, "type": "bf16", "out": "bf16", "pad": 0},
    ]


def _size(rng, lo, hi):
    """A size from lo to hi, spread over its logarithm; one in two is a multiple of 64."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and hi >= 64:
        v = max(64, (v + 32) // 64 * 64)
    return max(lo, min(hi, v))


def _rows(rng, hi):
    return max(1, min(hi, int(round(math.exp(rng.uniform(0.0, math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "gate", "w4", "w4"])
    if op == "norm":
        return {"op": op, "m": _rows(rng, 8192), "k": _size(rng, 64, 16384), "type": rng.choice(["bf16", "f16", "f32"]),
                "residual": rng.random() < 0.7, "pad": rng.choice([0, 0, 8, 5])}
    if op == "gate":
        return {"op": op, "m": _rows(rng, 4096), "f": _size(rng, 64, 16384), "type": rng.choice(["bf16", "f16", "f32"])}
    case = {"op": op, "m": _rows(rng, 4096), "n": _size(rng, 64, 16384), "k": _size(rng, 64, 16384), "group": rng.choice([32, 64, 128]),
            "zeros": rng.random() < 0.5, "type": rng.choice(["bf16", "f16", "e4m3"]), "pad": rng.choice([0, 0, 16, 3])}
    case["out"] = case["type"] if case["type"] != "e4m3" else rng.choice(["bf16", "f16"])
    case["m"] = max(1, min(case["m"], 4096 * 16384 * 4096 // (case["n"] * case["k"])))
    return case


def work(case):
    m, t = case["m"], SIZE[case["type"]]
    if case["op"] == "norm":
        mk = m * case["k"]
        res = 2 if case["residual"] else 0       # the residual is read and the sum is written
        return {"bytes": mk * t * (1 + res) + case["k"] * t + mk + 4 * m, "flops": 6 * mk}
    if case["op"] == "gate":
        mf = m * case["f"]
        return {"bytes": 2 * mf * t + mf + 4 * m, "flops": 6 * mf}
    n, k = case["n"], case["k"]
    groups = -(-k // case["group"])
    weights = n * -(-k // 2) + 2 * n * groups + (-(-n * groups // 2) if case["zeros"] else 0)
    return {"bytes": weights + m * k * t + (4 * m if case["type"] == "e4m3" else 0) + m * n * SIZE[case["out"]], "flops": 2 * m * n * k}


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
    n, k, group = case["n"], case["k"], case["group"]
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
    s = {"q": (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous(), "s": scale.to(TYPES[case["out"]]),
         "z": zero.to(torch.uint8) if case["zeros"] else None, "xs": None}
    if case["type"] == "e4m3":
        x = _stream(g, m, k, case["pad"], torch.float32)
        s["xs"] = x.abs().amax(-1).clamp_min(1e-6) / E4M3_MAX
        s["x"] = (torch.nn.functional.pad(x, (0, case["pad"])) / s["xs"][:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(dtype)[:, :k]
    else:
        s["x"] = _stream(g, m, k, case["pad"], dtype)
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
        else:
            s["matrix"] = sw.W4Matrix(s["q"], s["s"], s["z"], k=case["k"], group=case["group"])
            s["out"] = torch.empty(m, case["n"], dtype=TYPES[case["out"]], device="cuda")
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
        return state["matrix"](state["x"], state["xs"], out=state["out"])
    return {"norm": _norm, "gate": _gate, "w4": _w4}[case["op"]](state, case)


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


def _w4(state, case):
    n, k, group = case["n"], case["k"], case["group"]
    q = torch.stack([state["q"] & 15, state["q"] >> 4], -1).view(n, -1)[:, :k].float()
    scale = state["s"].float().repeat_interleave(group, 1)[:, :k]
    zero = state["z"].float().repeat_interleave(group, 1)[:, :k] if case["zeros"] else 8.0
    y = state["x"].float() @ (scale * (q - zero)).t()
    if state["xs"] is not None:
        y = y * state["xs"][:, None]
    return y.to(TYPES[case["out"]])


# ---- the same in 64 bits -----------------------------------------------------------------------------------------

def exact(case, seed):
    s = _inputs(case, seed)
    d = torch.float64
    if case["op"] == "norm":
        total = s["x"].to(d) if s["r"] is None else s["x"].to(d) + s["r"].to(d)
        values = total / torch.sqrt(torch.einsum("mk,mk->m", total, total) / case["k"] + EPS)[:, None] * s["w"].to(d)
    elif case["op"] == "gate":
        gate, up = s["gu"].to(d).split(case["f"], 1)
        values = gate * torch.special.expit(gate) * up
    else:
        # group by group: y = xs * sum_g S_g * (x_g . Q_g - Z_g * sum(x_g))
        n, k, group = case["n"], case["k"], case["group"]
        y = torch.zeros(case["m"], n, dtype=d, device="cuda")
        nibbles = torch.empty(n, 2 * s["q"].shape[1], dtype=d, device="cuda")
        nibbles[:, 0::2] = (s["q"] % 16).to(d)
        nibbles[:, 1::2] = (s["q"] // 16).to(d)
        x = s["x"].to(d)
        for i in range(-(-k // group)):
            a, b = i * group, min(k, (i + 1) * group)
            zero = 8.0 if s["z"] is None else s["z"][:, i].to(d)[:, None]
            y.addmm_(x[:, a:b], ((nibbles[:, a:b] - zero) * s["s"][:, i].to(d)[:, None]).t())
        return y if s["xs"] is None else y * s["xs"].to(d)[:, None]
    scale = torch.maximum(values.abs().max(1).values / E4M3_MAX, torch.full((case["m"],), MIN_SCALE, dtype=d, device="cuda"))
    out = (values / scale[:, None], scale)
    return out + (total,) if case["op"] == "norm" and s["r"] is not None else out
