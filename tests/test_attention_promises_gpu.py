"""What the attention operators' documentation promises beyond their formulas: the codes of 8-bit rows, every row counted once, what is refused."""
import math

import pytest
import torch

import paper_1202_3173_b200 as sw
from paper_1202_3173_b200 import StrassenError, binding

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


def ints(*x):
    return [torch.tensor(v, dtype=torch.int32, device="cuda") for v in x]


def stored(v, page=64):
    """(codes, scales) of rows v (tokens, kv, d) that were stored unturned, as keys and as values."""
    tokens, kv, d = v.shape
    pages = -(-tokens // page)
    cache = sw.PagedCache.empty(pages, kv, d, page, E4M3)
    table, lengths, offsets = ints([list(range(pages))], [tokens], [0, tokens])
    sw.rotate_append(None, v, v, cache, table, lengths, None, offsets)
    out = []
    for store, scales in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        out.append((store.view(torch.uint8).transpose(1, 2).flatten(0, 1)[:tokens], scales.transpose(1, 2).flatten(0, 1)[:tokens]))
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kv,d", [(8, 128), (3, 80), (1, 16)])
def test_rows_in_8_bits_are_the_rounded_quotients(kv, d, dtype):
    """Rows that do not turn: codes and scales are those of the division in 32 bits, bit for bit: random rows, and rows of each largest mantissa with every mantissa
    below, among which are quotients on and next to the borders between two codes."""
    g = torch.Generator("cuda").manual_seed(d)
    rows = [torch.randn(20000 // kv * kv, d, device="cuda", generator=g).to(dtype)]
    bits = 7 if dtype is torch.bfloat16 else 10
    mantissas = 1 + torch.arange(2 ** bits, device="cuda") / 2 ** bits
    for e in range(-8, 2):
        x = torch.empty(2 ** bits, d, device="cuda").uniform_(generator=g)
        x = mantissas[(x * 2 ** bits).long().clamp_max(2 ** bits - 1)] * 2.0 ** e
        x[:, 0] = 4 * mantissas
        rows.append(x.to(dtype))
    rows.append(torch.zeros(1, d, device="cuda", dtype=dtype))
    rows.append(torch.full((1, d), torch.finfo(dtype).max, device="cuda", dtype=dtype))
    rows.append(torch.full((1, d), torch.finfo(dtype).smallest_normal, device="cuda", dtype=dtype))
    rows.append(torch.full((1, d), 1.0, device="cuda", dtype=dtype).index_fill_(1, torch.tensor([d // 2], device="cuda"), math.inf))
    v = torch.cat(rows)
    v = v[:v.shape[0] // kv * kv].view(-1, kv, d) if kv > 1 else v[:, None]
    # divided in 64 bits and rounded to 32: a tensor over a number is the product with its reciprocal in torch, which is not always the rounded quotient
    scale = (v.double().abs().amax(-1) / 448).float().clamp_min(2.0 ** -64)
    want = (v.double() / scale.double()[..., None]).float().to(E4M3)
    for codes, scales in stored(v):
        assert torch.equal(scales, scale)
        nan = torch.isnan(want.float())
        assert torch.equal(codes[~nan], want.view(torch.uint8)[~nan]) and bool(((codes[nan] & 127) == 127).all())
