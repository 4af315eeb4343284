"""Cases of the attention operators of a served model: rotary embedding with the storing of keys and values into a paged cache,
attention of one new token a sequence over that cache, and attention of prompts over it.

Every operator is here in its plain form (32-bit torch operations, rounded once at the end; 64 bits for the angles), in 64 bits
(``exact``), and, with ``own`` set, as the calls of this package that a user makes.

Row j of sequence b lies in page ``table[b][j // page]``, slot ``j % page``.  ``lengths[b]`` counts the sequence's rows with the new ones, which
are the last ``offsets[b + 1] - offsets[b]`` (without offsets: one).
"""
import math
import random

import torch

own = False

E4M3_MAX = 448.0
MIN_SCALE = 2.0 ** -64       # smallest scale of an 8-bit row: a row of zeros is zeros with this scale
THETA = 500000.0
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f16": 2, "e4m3": 1}


def listed():
    return [
        # one new token of one request, bf16 cache: the smallest call of generation
        {"name": "append 1 token 32+8x128 bf16", "op": "append", "batch": 1, "new": 1, "past": 700, "heads": 32, "kv": 8, "d": 128, "page": 64, "type": "bf16", "cache": "bf16",
         "interleaved": False, "rotary": 128},
        # ragged prompts of a batch, most of them behind cached ones, 80-wide heads of which a part turns, neighbours as pairs
        {"name": "append 9x301 tokens 12+12x80 f16", "op": "append", "batch": 9, "new": 301, "past": 2000, "heads": 12, "kv": 12, "d": 80, "page": 16, "type": "f16", "cache": "f16",
         "interleaved": True, "rotary": 64},
        # a long prompt into an 8-bit cache
        {"name": "append 16384 tokens 32+8x128 e4m3", "op": "append", "batch": 1, "new": 16384, "past": 0, "heads": 32, "kv": 8, "d": 128, "page": 64, "type": "bf16", "cache": "e4m3",
         "interleaved": False, "rotary": 128},
        # one request, early in its answer: latency counts
        {"name": "decode 1x1000 32/8x128 bf16", "op": "decode", "batch": 1, "length": 1000, "heads": 32, "kv": 8, "d": 128, "page": 64, "type": "bf16", "cache": "bf16", "window": 0},
        # one request with a very long context: the cache's length has to be split over the GPU
        {"name": "decode 1x131071 32/8x128 bf16", "op": "decode", "batch": 1, "length": 131071, "heads": 32, "kv": 8, "d": 128, "page": 16, "type": "bf16", "cache": "bf16", "window": 0},
        # a small batch without grouped heads, odd width, pages that end inside tiles
        {"name": "decode 33x4099 12/12x80 f16", "op": "decode", "batch": 33, "length": 4099, "heads": 12, "kv": 12, "d": 80, "page": 32, "type": "f16", "cache": "f16", "window": 0},
        # a batch over an 8-bit cache, seven heads to a key head
        {"name": "decode 64x8192 28/4x128 e4m3", "op": "decode", "batch": 64, "length": 8192, "heads": 28, "kv": 4, "d": 128, "page": 64, "type": "bf16", "cache": "e4m3", "window": 0},
        # a large batch of long requests
        {"name": "decode 32x32768 64/8x128 bf16", "op": "decode", "batch": 32, "length": 32768, "heads": 64, "kv": 8, "d": 128, "page": 128, "type": "bf16", "cache": "bf16", "window": 0},
        # one ordinary prompt
        {"name": "prompt 1x512 32/8x128 bf16", "op": "prompt", "batch": 1, "new": 512, "past": 0, "heads": 32, "kv": 8, "d": 128, "page": 64, "type": "bf16", "cache": "bf16", "window": 0},
        # packed prompts of different odd lengths, some behind cached ones, in pages shorter than a tile
        {"name": "prompt 7x2049 28/4x80 f16", "op": "prompt", "batch": 7, "new": 2049, "past": 1500, "heads": 28, "kv": 4, "d": 80, "page": 16, "type": "f16", "cache": "f16", "window": 0},
        # the next parts of long prompts, each token seeing a window
        {"name": "prompt 4x2048 behind 16384 64/8x64 window 4096 bf16", "op": "prompt", "batch": 4, "new": 2048, "past": 16384, "heads": 64, "kv": 8, "d": 64, "page": 64, "type": "bf16",
         "cache": "bf16", "window": 4096},
        # a long prompt
        {"name": "prompt 1x16384 32/8x128 bf16", "op": "prompt", "batch": 1, "new": 16384, "past": 0, "heads": 32, "kv": 8, "d": 128, "page": 64, "type": "bf16", "cache": "bf16", "window": 0},
    ]


def _size(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "decode", "decode", "prompt", "prompt"])
    kv = rng.choice([1, 2, 4, 5, 8, 12])
    group = rng.choice([1, 1, 2, 3, 4, 4, 7, 8, 8, 16])
    d = rng.choice([64, 64, 80, 96, 112, 128, 128, 128, 128])
    case = {"op": op, "batch": _size(rng, 1, 128), "heads": kv * group, "kv": kv, "d": d, "page": rng.choice([16, 32, 64, 128]), "type": rng.choice(["bf16", "f16"])}
    if op == "append":
        case.update(cache=rng.choice([case["type"], "e4m3"]), new=_size(rng, 1, 16384), past=rng.choice([0, _size(rng, 1, 8192)]), interleaved=rng.random() < 0.3,
                    rotary=rng.choice([d, d, 32]))
        case["batch"] = max(1, min(case["batch"], 16384 * 48 * 128 // ((case["new"] + case["past"]) * (case["heads"] + 2 * kv) * d)))
        case["new"] = max(1, min(case["new"], 16384 * 48 * 128 // (case["batch"] * (case["heads"] + 2 * kv) * d)))
    elif op == "decode":
        case.update(cache=rng.choice([case["type"], "e4m3"]), length=_size(rng, 16, 131072), window=rng.choice([0, 0, 0, _size(rng, 16, 4096)]))
        case["batch"] = max(1, min(case["batch"], 32 * 32768 * 8 * 128 // (case["length"] * kv * d)))
        case["length"] = max(1, min(case["length"], 32 * 32768 * 8 * 128 // (case["batch"] * kv * d)))
    else:
        case.update(cache=case["type"], new=_size(rng, 2, 16384), past=rng.choice([0, 0, _size(rng, 1, 16384)]), window=rng.choice([0, 0, 0, _size(rng, 16, 4096)]))
        case["batch"] = min(case["batch"], 32)
        while _pairs_bound(case) * case["heads"] * d > 16384 * 16384 // 2 * 32 * 128 or case["batch"] * (case["new"] + case["past"]) * kv * d > 32 * 32768 * 8 * 128:
            if case["batch"] > 1:
                case["batch"] //= 2
            elif case["past"] > case["new"]:
                case["past"] //= 2
            else:
                case["new"] = max(2, case["new"] // 2)
    return case


def _pairs_bound(case):
    return case["batch"] * case["new"] * (case["new"] / 2 + case["past"])


# ---- lengths ---------------------------------------------------------------------------------------------------

def _ragged(case):
    """(lengths, counts) of the sequences, from the sizes alone, so that every seed's inputs are as large: the first has the full length, the others between a
    quarter (past rows: none) of it and all."""
    rng = random.Random(case["batch"] * 7919 + case["d"])
    lengths, counts = [], []
    for b in range(case["batch"]):
        part, behind = (1.0, 1.0) if b == 0 else (rng.uniform(0.25, 1.0), rng.uniform(0.0, 1.0))
        if case["op"] == "decode":
            counts.append(1)
            lengths.append(max(1, int(case["length"] * part)))
        else:
            counts.append(max(1, int(case["new"] * part)))
            lengths.append(counts[-1] + int(case["past"] * behind))
    return lengths, counts


def _visible(case):
    """(query, row) pairs that are seen, over all sequences."""
    window, total = case.get("window", 0), 0
    for length, count in zip(*_ragged(case)):
        first = length - count                      # the position of the first new token sees first + 1 rows
        if not window or length <= window:
            total += count * first + count * (count + 1) // 2
        else:
            full = min(count, length - max(first, window))          # queries that see the whole window
            short = count - full
            total += full * window + short * first + short * (short + 1) // 2
    return total


def work(case):
    lengths, counts = _ragged(case)
    heads, kv, d, t, c = case["heads"], case["kv"], case["d"], SIZE[case["type"]], SIZE[case["cache"]]
    row = kv * (d * c + (4 if case["cache"] == "e4m3" else 0))            # a key or a value row of all heads in the cache
    new = sum(counts)
    if case["op"] == "append":
        return {"bytes": new * (2 * heads * d * t + 2 * kv * d * t + 2 * row) + 4 * case["rotary"] // 2, "flops": new * (heads + kv) * case["rotary"] * 3}
    window = case["window"]
    seen = sum(min(n, window + m - 1) if window else n for n, m in zip(lengths, counts))
    pairs = _visible(case)
    return {"bytes": 2 * seen * row + 2 * new * heads * d * t, "flops": 4 * pairs * heads * d}


# ---- inputs ----------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows_to_8_bits(v):
    s = (v.abs().amax(-1) / E4M3_MAX).clamp_min(MIN_SCALE)
    return (v / s[..., None]).to(torch.float8_e4m3fn), s


def _inputs(case, seed):
    g, lengths, counts = _generator(seed), *_ragged(case)
    batch, heads, kv, d, page, dtype = case["batch"], case["heads"], case["kv"], case["d"], case["page"], TYPES[case["type"]]
    needed = [-(-n // page) for n in lengths]
    pages = sum(needed) + 3
    # pages as a server has handed them out: in no order; behind the last one of a sequence the table holds no page
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
    table = torch.full((batch, max(needed)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(needed):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    s = {"table": table.cuda(), "lengths": torch.tensor(lengths, dtype=torch.int32).cuda(), "table_host": table.tolist(), "lengths_host": lengths, "counts_host": counts}
    offsets = [0]
    for n in counts:
        offsets.append(offsets[-1] + n)
    s["offsets_host"] = offsets
    s["offsets"] = torch.tensor(offsets, dtype=torch.int32).cuda() if case["op"] == "prompt" or max(counts) > 1 else None
    # channels of different size, as keys have them, and a direction that queries share, along which the first row of a sequence lies: most queries
    # look at it
    gain = 1 + 3 * (torch.rand(kv, 1, d, device="cuda", generator=g) < 0.03)
    shared = 0.4 * torch.randn(kv, 1, d, device="cuda", generator=g)
    if case["op"] == "append":
        # one product's output row holds a token's queries, keys and values
        qkv = torch.randn(offsets[-1], heads + 2 * kv, d, device="cuda", generator=g)
        qkv[:, heads:heads + kv] *= gain[:, 0]
        qkv = qkv.to(dtype)
        s["q"], s["k"], s["v"] = qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:]
        s["frequencies"] = (THETA ** (-torch.arange(0, case["rotary"], 2, dtype=torch.float64) / case["rotary"])).float().cuda()
        s["cache"] = [torch.zeros(pages, kv, page, d, dtype=TYPES[case["cache"]], device="cuda") for _ in range(2)]
        s["scales"] = [torch.zeros(pages, kv, page, device="cuda") if case["cache"] == "e4m3" else None for _ in range(2)]
        return s
    q = torch.randn(offsets[-1], kv, heads // kv, d, device="cuda", generator=g) + shared
    s["q"] = q.view(offsets[-1], heads, d).to(dtype)
    s["cache"], s["scales"] = [], []
    for which in range(2):
        store = torch.empty(pages, kv, page, d, dtype=TYPES[case["cache"]], device="cuda")
        scales = torch.empty(pages, kv, page, device="cuda") if case["cache"] == "e4m3" else None
        part = max(1, (1 << 26) // (kv * page * d))
        for i in range(0, pages, part):
            v = torch.randn(min(part, pages - i), kv, page, d, device="cuda", generator=g)
            if which == 0:
                v *= gain
            if case["cache"] == "e4m3":
                store[i:i + part], scales[i:i + part] = _rows_to_8_bits(v)
            else:
                store[i:i + part] = v
        if which == 0:
            first = table[:, 0].long().cuda()
            v = (3 * shared[:, 0]).expand(batch, kv, d)
            if case["cache"] == "e4m3":
                v, scale = _rows_to_8_bits(v)
                scales[first, :, 0] = scale
                store.view(torch.uint8)[first, :, 0] = v.view(torch.uint8)
            else:
                store[first, :, 0] = v.to(store.dtype)
        s["cache"].append(store)
        s["scales"].append(scales)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        import paper_1202_3173_b200 as sw
        # the cache's handle and the buffers that a serving program keeps
        s["paged"] = sw.PagedCache(s["cache"][0], s["cache"][1], s["scales"][0], s["scales"][1])
        s["out"] = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    return s


# ---- one pass --------------------------------------------------------------------------------------------------

def run(state):
    case = state["case"]
    if own:
        import paper_1202_3173_b200 as sw
        if case["op"] == "append":
            q = sw.rotate_append(state["q"], state["k"], state["v"], state["paged"], state["table"], state["lengths"], frequencies=state["frequencies"],
                                 offsets=state["offsets"], interleaved=case["interleaved"], out=state["out"])
            return _updated(state, q)
        if case["op"] == "decode":
            return sw.decode_attention(state["q"], state["paged"], state["table"], state["lengths"], window=case["window"], out=state["out"])
        return sw.prompt_attention(state["q"], state["paged"], state["table"], state["lengths"], state["offsets"], window=case["window"], out=state["out"])
    return _append(state, case) if case["op"] == "append" else _attention(state, case)


def _updated(state, q):
    (k, v), (ks, vs) = state["cache"], state["scales"]
    return (q, k, v) if ks is None else (q, k, v, ks, vs)


def _where(state, case):
    """(positions, page, slot) of the new tokens."""
    n = state["q"].shape[0]
    token = torch.arange(n, device="cuda")
    if state["offsets"] is None:
        b, first, end = token, token, token + 1
    else:
        b = torch.searchsorted(state["offsets"], token.to(torch.int32), right=True) - 1
        first, end = state["offsets"][b], state["offsets"][b + 1]
    p = state["lengths"][b] - (end - first) + (token - first)
    return p, state["table"][b, p // case["page"]].long(), p % case["page"]


def _turn(x, cos, sin, rotary, interleaved):
    x = x.float()
    if interleaved:
        a, b = x[..., 0:rotary:2], x[..., 1:rotary:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :rotary // 2], x[..., rotary // 2:rotary]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., rotary:]], -1)


def _append(state, case):
    p, page, slot = _where(state, case)
    angle = p.double()[:, None] * state["frequencies"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    q = _turn(state["q"], cos, sin, case["rotary"], case["interleaved"]).to(state["q"].dtype)
    rows = _turn(state["k"], cos, sin, case["rotary"], case["interleaved"]), state["v"].float()
    for store, scales, v in zip(state["cache"], state["scales"], rows):
        if case["cache"] == "e4m3":
            v, scale = _rows_to_8_bits(v)
            scales[page, :, slot] = scale
            store.view(torch.uint8)[page, :, slot] = v.view(torch.uint8)
        else:
            store[page, :, slot] = v.to(store.dtype)
    return _updated(state, q)


def _sequence(state, case, b, which, dtype):
    """Keys or values of sequence b: (kv heads, length, d)."""
    n, page = state["lengths_host"][b], case["page"]
    pages = state["table"][b, :-(-n // page)].long()
    rows = state["cache"][which][pages].to(dtype)
    if case["cache"] == "e4m3":
        rows = rows * state["scales"][which][pages].to(dtype)[..., None]
    return rows.transpose(0, 1).flatten(1, 2)[:, :n]


def _attention(state, case):
    heads, kv, d, window = case["heads"], case["kv"], case["d"], case["window"]
    out = torch.empty_like(state["q"])
    for b, (n, m) in enumerate(zip(state["lengths_host"], state["counts_host"])):
        k, v = _sequence(state, case, b, 0, torch.float32), _sequence(state, case, b, 1, torch.float32)
        row = torch.arange(n, device="cuda")
        step = max(1, (1 << 28) // (heads * n))
        for i in range(0, m, step):
            at = state["offsets_host"][b] + i
            count = min(step, m - i)
            first, last = n - m + i, n - m + i + count              # positions of these queries
            lo = max(0, first - window + 1) if window else 0
            q = state["q"][at:at + count].float().view(count, kv, heads // kv, d).permute(1, 2, 0, 3).reshape(kv, -1, d)
            s = (q @ k[:, lo:last].transpose(1, 2)) * d ** -0.5
            s = s.view(kv, heads // kv, count, last - lo)
            if count > 1 or window:
                p = torch.arange(first, last, device="cuda")[:, None]
                hidden = row[lo:last] > p
                if window:
                    hidden = hidden | (row[lo:last] <= p - window)
                s = s.masked_fill(hidden, -math.inf)
            s = (s - s.amax(-1, keepdim=True)).exp()
            o = (s.view(kv, -1, last - lo) @ v[:, lo:last]).view(kv, heads // kv, count, d) / s.sum(-1, keepdim=True)
            out[at:at + count] = o.permute(2, 0, 1, 3).reshape(count, heads, d).to(out.dtype)
    return out


# ---- the same in 64 bits -----------------------------------------------------------------------------------------

def _exact_append(s, case):
    d64, r, half = torch.float64, case["rotary"], case["rotary"] // 2
    position = torch.cat([torch.arange(n - m, n) for n, m in zip(s["lengths_host"], s["counts_host"])]).to(d64).cuda()
    turn = torch.polar(torch.ones(position.shape[0], half, dtype=d64, device="cuda"), position[:, None] * s["frequencies"].to(d64))[:, None]
    turned = []
    for name in ("q", "k"):
        x = s[name].to(d64).clone()
        pairs = x[..., :r].unflatten(-1, (half, 2)) if case["interleaved"] else x[..., :r].unflatten(-1, (2, half)).transpose(-1, -2)
        pairs = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        x[..., :r] = pairs.flatten(-2) if case["interleaved"] else pairs.transpose(-1, -2).flatten(-2)
        turned.append(x)
    place = []
    for b, (n, m) in enumerate(zip(s["lengths_host"], s["counts_host"])):
        pages = torch.tensor(s["table_host"][b])
        place.append(pages.repeat_interleave(case["page"])[n - m:n] * case["page"] + torch.arange(n - m, n) % case["page"])
    place = torch.cat(place).cuda()
    out, scales = [turned[0]], []
    for v in (turned[1], s["v"].to(d64)):
        pages = s["cache"][0].shape[0]
        store = torch.zeros(pages * case["page"], case["kv"], case["d"], dtype=d64, device="cuda")
        if case["cache"] == "e4m3":
            scale = torch.clamp(torch.linalg.vector_norm(v, math.inf, dim=-1) / E4M3_MAX, min=MIN_SCALE)
            v = v / scale[..., None]
            scales.append(torch.zeros(pages * case["page"], case["kv"], dtype=d64, device="cuda").index_copy_(0, place, scale).unflatten(0, (pages, case["page"])).transpose(1, 2))
        out.append(store.index_copy_(0, place, v).unflatten(0, (pages, case["page"])).transpose(1, 2))
    return tuple(out + scales)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "append":
        return _exact_append(s, case)
    d64, kv, group, d, window = torch.float64, case["kv"], case["heads"] // case["kv"], case["d"], case["window"]
    out = torch.empty(s["q"].shape, dtype=d64, device="cuda")
    for b, (n, m) in enumerate(zip(s["lengths_host"], s["counts_host"])):
        where = torch.tensor(s["table_host"][b]).cuda().repeat_interleave(case["page"])[:n].long() * kv * case["page"] + torch.arange(n, device="cuda") % case["page"]
        for h in range(kv):
            rows = []
            for store, scale in zip(s["cache"], s["scales"]):
                x = store.view(-1, d)[where + h * case["page"]].to(d64)
                rows.append(x if scale is None else x * scale.view(-1)[where + h * case["page"]].to(d64)[:, None])
            step = max(1, (1 << 27) // (group * n))
            for i in range(0, m, step):
                at = slice(s["offsets_host"][b] + i, s["offsets_host"][b] + min(m, i + step))
                score = torch.einsum("qgd,jd->qgj", s["q"][at, h * group:(h + 1) * group].to(d64), rows[0]) / math.sqrt(d)
                behind = torch.arange(n - m + i, n - m + min(m, i + step), device="cuda")[:, None, None] - torch.arange(n, device="cuda")     # how far a row lies back
                score = torch.where((behind >= 0) & ((behind < window) if window else True), score, torch.full((), -math.inf, dtype=d64, device="cuda"))
                out[at, h * group:(h + 1) * group] = torch.einsum("qgj,jd->qgd", (score - torch.logsumexp(score, -1, keepdim=True)).exp_(), rows[1])
    return out
