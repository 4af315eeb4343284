"""Attention operators against plain implementations in 64 bits: rotary embedding and the paged cache, one new token, prompts.

Tolerances.  u is half a step of the output's type.  A result is rounded once: u |o|.  The softmax's weights are rounded once to 16 bits before the product with the
values: u A with A = sum of weight |value|; and their exponents err by the scores' error, E = (d + 8) 2^-23 max_j sum_i |q_i k_ij| scale (a sum of d products
in 32 bits), which changes a weight and the sum of weights by a factor 1 + E each.  Exponentials and the sums of up to 2^17 terms in 32 bits: 2^-18.  Together
u |o| + (u + 2 E + 2^-18) A.  In 8 bits the cache's values are what they stand for, exactly; beside them weights are f16 whatever q's type is (2^-11, not more than u).
"""
import math

import pytest
import torch

import paper_1202_3173_b200 as sw
from paper_1202_3173_b200 import StrassenError, binding

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def eight_bits(v):
    s = (v.abs().amax(-1) / 448).clamp_min(2.0 ** -64)
    return (v / s[..., None]).to(E4M3), s


class Case:
    """Sequences of these lengths in a cache whose other slots hold NaN."""

    def __init__(self, lengths, counts=None, heads=8, kv=2, d=128, page=16, dtype=torch.bfloat16, cache=None, seed=0, layout="pages", spread=1.0):
        g = gen(seed)
        cache = cache or dtype
        self.lengths_host, self.counts = list(lengths), list(counts or [1] * len(lengths))
        self.heads, self.kv, self.d, self.page, self.dtype = heads, kv, d, page, dtype
        batch, width = len(lengths), max([1] + [-(-n // page) for n in lengths])
        pages = sum(-(-n // page) for n in lengths) + 2
        order = torch.randperm(pages, device="cuda", generator=g).tolist()
        self.table = torch.full((batch, width), -1, dtype=torch.int32)
        self.k64, self.v64 = [], []
        shape = {"pages": (pages, kv, page, d), "rows": (pages, page, kv, d), "heads": (kv, pages, page, d)}[layout]
        def memory():
            t = torch.full(shape, math.nan, device="cuda").to(cache)
            return {"pages": t, "rows": t.transpose(1, 2), "heads": t.transpose(0, 1)}[layout]
        k, v = memory(), memory()
        ks, vs = (torch.full((pages, kv, page), math.nan, device="cuda") if cache == E4M3 else None for _ in range(2))
        at = 0
        for b, n in enumerate(lengths):
            used = -(-n // page)
            mine = order[at:at + used]
            self.table[b, :used] = torch.tensor(mine, dtype=torch.int32)
            at += used
            for store, scales, into in ((k, ks, self.k64), (v, vs, self.v64)):
                x = torch.randn(n, kv, d, device="cuda", generator=g) * spread
                if cache == E4M3:
                    x, s = eight_bits(x)
                    into.append(x.double() * s.double()[..., None])
                else:
                    x = x.to(cache)
                    into.append(x.double())
                for i, p in enumerate(mine):
                    part = x[i * page:(i + 1) * page].transpose(0, 1)
                    (store.view(torch.uint8) if cache == E4M3 else store)[p, :, :part.shape[1]] = part.view(torch.uint8) if cache == E4M3 else part
                    if cache == E4M3:
                        scales[p, :, :part.shape[1]] = s[i * page:(i + 1) * page].t()
        self.cache = sw.PagedCache(k, v, ks, vs)
        self.table = self.table.cuda()
        self.lengths = torch.tensor(self.lengths_host, dtype=torch.int32, device="cuda")
        offsets = [0]
        for n in self.counts:
            offsets.append(offsets[-1] + n)
        self.offsets_host = offsets
        self.offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        self.q = (torch.randn(offsets[-1], heads, d, device="cuda", generator=g) * spread).to(dtype)

    def reference(self, scale=None, window=0, dead=None):
        """(result, tolerance) in 64 bits.  dead: rows that nothing sees, by sequence."""
        scale = self.d ** -0.5 if scale is None else scale
        out = torch.zeros(self.q.shape, dtype=torch.float64, device="cuda")
        tol = torch.zeros_like(out)
        u = HALF_STEP[self.dtype]
        for b, (n, m) in enumerate(zip(self.lengths_host, self.counts)):
            rows = slice(self.offsets_host[b], self.offsets_host[b + 1])
            q = self.q[rows].double()
            p = torch.arange(n - m, n, device="cuda")
            j = torch.arange(n, device="cuda")
            seen = j <= p[:, None]
            if window:
                seen &= j > p[:, None] - window
            for h in range(self.heads):
                k, v = (x[b][:, h // (self.heads // self.kv)] for x in (self.k64, self.v64))
                s = (q[:, h] @ k.t()) * scale
                s = torch.where(seen, s, torch.full_like(s, -math.inf))
                w = torch.where(seen.any(1, keepdim=True), torch.softmax(s, 1), torch.zeros_like(s)) if n else s
                e = torch.where(seen, (q[:, h].abs() @ k.abs().t()) * abs(scale), torch.zeros_like(s)).amax(1, keepdim=True) * (self.d + 8) * 2.0 ** -23 if n else 0
                out[rows, h] = w @ v
                tol[rows, h] = u * out[rows, h].abs() + (u + 2 * e + 2.0 ** -18) * (w @ v.abs())
        return out, tol


def close(got, want, tol):
    assert bool(torch.isfinite(got).all())
    if got.numel() == 0:
        return
    worst = ((got.double() - want).abs() / (tol + 1e-30))
    assert float(worst.max()) <= 1, "%g of the tolerance at %s" % (float(worst.max()), (worst == worst.max()).nonzero()[0].tolist())


# ---- one new token ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("page", [8, 16, 64, 256])
@pytest.mark.parametrize("lengths", [[1], [1, 2, 15, 16, 17], [127, 128, 129, 63, 64, 65], [1000, 3, 777, 0, 2049], [5000]])
def test_decode_lengths(lengths, page):
    c = Case(lengths, page=page, seed=page + len(lengths))
    close(sw.decode_attention(c.q, c.cache, c.table, c.lengths), *c.reference())


@pytest.mark.parametrize("dtype,cache", [(torch.bfloat16, None), (torch.float16, None), (torch.bfloat16, E4M3), (torch.float16, E4M3)])
@pytest.mark.parametrize("heads,kv,d", [(1, 1, 128), (4, 4, 64), (6, 2, 80), (7, 1, 128), (8, 1, 96), (28, 4, 128), (12, 1, 112), (16, 1, 64), (20, 1, 48), (40, 2, 128), (3, 3, 16)])
def test_decode_heads_and_types(heads, kv, d, dtype, cache):
    c = Case([300, 41, 129], heads=heads, kv=kv, d=d, dtype=dtype, cache=cache, page=32, seed=heads)
    close(sw.decode_attention(c.q, c.cache, c.table, c.lengths), *c.reference())


def test_decode_head_sizes_of_16_bits():
    for d in (8, 24, 40, 56, 72, 88, 104, 120):
        c = Case([70, 9], heads=4, kv=2, d=d, dtype=torch.float16, seed=d)
        close(sw.decode_attention(c.q, c.cache, c.table, c.lengths), *c.reference())


@pytest.mark.parametrize("window", [1, 2, 16, 100, 129, 5000, 2 ** 40])
@pytest.mark.parametrize("cache", [None, E4M3])
def test_decode_window(window, cache):
    c = Case([1, 99, 100, 101, 1500], cache=cache, page=16, seed=window % 1000)
    close(sw.decode_attention(c.q, c.cache, c.table, c.lengths, window=window), *c.reference(window=window))


@pytest.mark.parametrize("layout", ["rows", "heads"])
@pytest.mark.parametrize("cache", [None, E4M3])
def test_decode_other_orders_of_the_cache(layout, cache):
    c = Case([333, 65], layout=layout, cache=cache, heads=6, kv=3)
    close(sw.decode_attention(c.q, c.cache, c.table, c.lengths), *c.reference())


def test_decode_long_and_many():
    for lengths, kv, cache in (([40000], 1, None), ([1 + 37 * i % 700 for i in range(200)], 2, None), ([30000, 5, 20000], 2, E4M3)):
        c = Case(lengths, heads=4 * kv, kv=kv, page=64, cache=cache, seed=len(lengths))
        close(sw.decode_attention(c.q, c.cache, c.table, c.lengths), *c.reference())


@pytest.mark.parametrize("cache", [None, E4M3])
def test_decode_scores_far_apart(cache):
    """Scores of some hundreds, falling and rising along the sequence, and a negative scale."""
    c = Case([2000, 513], spread=6.0, cache=cache, dtype=torch.float16, seed=3)
    close(sw.decode_attention(c.q, c.cache, c.table, c.lengths, scale=0.02), *c.reference(scale=0.02))
    close(sw.decode_attention(c.q, c.cache, c.table, c.lengths, scale=-0.03), *c.reference(scale=-0.03))
    close(sw.decode_attention(c.q, c.cache, c.table, c.lengths, scale=0.0), *c.reference(scale=0.0))


def test_decode_many_small_weights_count():
    """One row far above 60000 others, whose weights are each below the smallest f16 number and together 1/600 of the whole."""
    n = 60000
    for cache in (None, E4M3):
        c = Case([n], heads=1, kv=1, d=64, dtype=torch.float16, cache=cache, page=256)
        c.q.zero_()
        c.q[..., 0] = 1.0
        k = torch.zeros(n, 1, 64, device="cuda")
        k[0, 0, 0] = 17.4
        v = torch.full((n, 1, 64), 2.0, device="cuda")
        v[0] = 1.0
        fill(c, 0, k, v)
        close(sw.decode_attention(c.q, c.cache, c.table, c.lengths, scale=1.0), *c.reference(scale=1.0))


def fill(c, b, k, v):
    """Sequence b's rows replaced."""
    for x, store, scales, into in ((k, c.cache.k, c.cache.k_scale, c.k64), (v, c.cache.v, c.cache.v_scale, c.v64)):
        n = x.shape[0]
        pages = c.table[b].long()[torch.arange(n, device="cuda") // c.page]
        slots = torch.arange(n, device="cuda") % c.page
        if scales is not None:
            x, s = eight_bits(x)
            into[b] = x.double() * s.double()[..., None]
            scales[pages, :, slots] = s
            store.view(torch.uint8)[pages, :, slots] = x.view(torch.uint8)
        else:
            x = x.to(store.dtype)
            into[b] = x.double()
            store[pages, :, slots] = x


def test_decode_values_of_very_different_rows_in_8_bits():
    """Value rows of 2^-60 and of 2^20 side by side, zeros among them."""
    n = 300
    c = Case([n], heads=2, kv=1, d=64, cache=E4M3)
    g = gen(5)
    v = torch.randn(n, 1, 64, device="cuda", generator=g) * torch.exp2(torch.randint(-60, 20, (n, 1, 1), device="cuda", generator=g).float())
    v[7] = 0
    fill(c, 0, torch.randn(n, 1, 64, device="cuda", generator=g), v)
    close(sw.decode_attention(c.q, c.cache, c.table, c.lengths), *c.reference())
    fill(c, 0, torch.randn(n, 1, 64, device="cuda", generator=g), torch.zeros(n, 1, 64, device="cuda"))
    assert not bool(sw.decode_attention(c.q, c.cache, c.table, c.lengths).any())


def test_decode_strided_and_misaligned_queries_and_results():
    c = Case([300, 41], heads=6, kv=2, d=80, dtype=torch.float16)
    want, tol = c.reference()
    buffer = torch.zeros(2, 6 * 83 + 5, dtype=torch.float16, device="cuda")
    q = torch.as_strided(buffer, (2, 6, 80), (6 * 83 + 5, 83, 1), 3)
    q.copy_(c.q)
    back = torch.full((2, 6 * 81 + 1), 7.0, dtype=torch.float16, device="cuda")
    out = torch.as_strided(back, (2, 6, 80), (6 * 81 + 1, 81, 1), 1)
    assert sw.decode_attention(q, c.cache, c.table, c.lengths, out=out) is out
    close(out, want, tol)
    assert bool((back[:, 0] == 7).all()) and bool((torch.as_strided(back, (2, 6), (6 * 81 + 1, 81), 81) == 7)[:, :5].all())
    # heads before rows
    q = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    close(sw.decode_attention(q, c.cache, c.table, c.lengths), want, tol)


@pytest.mark.parametrize("cache", [None, E4M3])
def test_pages_that_are_not_there_read_as_zeros(cache):
    c = Case([100, 100], cache=cache, page=16)
    for number in (-1, -2 ** 31, c.cache.pages, 2 ** 31 - 1):
        c.table[1, 2] = number
        c.k64[1][32:48] = 0
        c.v64[1][32:48] = 0
        close(sw.decode_attention(c.q, c.cache, c.table, c.lengths), *c.reference())
        c.q, c.counts, c.offsets_host = c.q[:2], [1, 1], [0, 1, 2]
        close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")), *c.reference())


def test_lengths_beyond_the_table_and_below_zero():
    c = Case([64, 64, 64], page=16)
    want, tol = c.reference()
    lengths = torch.tensor([2 ** 31 - 1, 64, -2 ** 31], dtype=torch.int32, device="cuda")
    got = sw.decode_attention(c.q, c.cache, c.table, lengths)
    close(got[:2], want[:2], tol[:2])
    assert not bool(got[2].any())
    one = torch.tensor([0, 1, 2, 3], dtype=torch.int32, device="cuda")
    got = sw.prompt_attention(c.q, c.cache, c.table, lengths, one)
    close(got[:2], want[:2], tol[:2])
    assert not bool(got[2].any())


def test_nothing_to_do():
    c = Case([5], page=16)
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    assert sw.decode_attention(c.q[:0], c.cache, c.table[:0], empty).shape == (0, 8, 128)
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    assert sw.prompt_attention(c.q[:0], c.cache, c.table[:0], empty, zero).shape == (0, 8, 128)
    assert not bool(sw.decode_attention(c.q, c.cache, c.table, zero).any())
    assert not bool(sw.decode_attention(c.q, c.cache, c.table[:, :0], c.lengths).any())


# ---- prompts --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("cache", [None, E4M3])
@pytest.mark.parametrize("page", [8, 16, 64, 128, 512])
@pytest.mark.parametrize("lengths,counts", [([1], [1]), ([7, 130, 1], [7, 130, 1]), ([128, 256, 127, 129], [128, 256, 127, 129]), ([700], [700]),
                                            ([500, 40, 1000, 0, 300], [3, 40, 129, 0, 17]), ([2000], [64])])
def test_prompt_lengths(lengths, counts, page, cache):
    c = Case(lengths, counts, page=page, seed=page, cache=cache)
    close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets), *c.reference())


@pytest.mark.parametrize("dtype,cache", [(torch.bfloat16, None), (torch.float16, None), (torch.bfloat16, E4M3), (torch.float16, E4M3)])
@pytest.mark.parametrize("heads,kv,d", [(1, 1, 128), (4, 4, 64), (6, 2, 80), (7, 1, 128), (8, 1, 96), (28, 4, 128), (12, 1, 112), (16, 1, 64), (20, 1, 48), (40, 2, 128), (3, 3, 16), (130, 1, 32)])
def test_prompt_heads_and_types(heads, kv, d, dtype, cache):
    c = Case([300, 41, 129], [200, 41, 5], heads=heads, kv=kv, d=d, dtype=dtype, cache=cache, page=32, seed=heads)
    close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets), *c.reference())


def test_prompt_head_sizes_of_16_bits():
    for d in (8, 24, 40, 56, 72, 88, 104, 120):
        c = Case([170, 9], [170, 3], heads=4, kv=2, d=d, dtype=torch.float16, seed=d)
        close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets), *c.reference())


@pytest.mark.parametrize("cache", [None, E4M3])
@pytest.mark.parametrize("window", [1, 2, 16, 100, 129, 300, 5000, 2 ** 40])
def test_prompt_window(window, cache):
    c = Case([1, 99, 100, 901, 1500], [1, 99, 7, 901, 300], page=16, heads=4, kv=2, seed=window % 1000, cache=cache)
    close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets, window=window), *c.reference(window=window))


@pytest.mark.parametrize("layout", ["rows", "heads"])
@pytest.mark.parametrize("cache", [None, E4M3])
def test_prompt_other_orders_of_the_cache(layout, cache):
    c = Case([333, 65], [333, 60], layout=layout, heads=6, kv=3, cache=cache)
    close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets), *c.reference())


@pytest.mark.parametrize("cache", [None, E4M3])
def test_prompt_long_and_many(cache):
    for lengths, counts, kv in (([3500], [3500], 1), ([1 + 37 * i % 200 for i in range(150)], None, 1), ([20000, 33], [100, 33], 2), ([300 + i for i in range(33)], [1 + 5 * i for i in range(33)], 1)):
        c = Case(lengths, counts or lengths, heads=4 * kv, kv=kv, page=64, seed=len(lengths), cache=cache)
        close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets), *c.reference())


@pytest.mark.parametrize("cache", [None, E4M3])
def test_prompt_scores_far_apart(cache):
    c = Case([1000, 513], [1000, 200], spread=6.0, dtype=torch.float16, seed=3, heads=4, kv=1, cache=cache)
    for scale in (0.02, -0.03, 0.0):
        close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets, scale=scale), *c.reference(scale=scale))
    # scores that rise by hundreds, so that what was added up before is scaled down again and again
    n = 1000
    k = torch.zeros(n, 1, 128, device="cuda")
    k[:, 0, 0] = torch.arange(n, device="cuda") * 0.25
    fill(c, 0, k, torch.randn(n, 1, 128, device="cuda", generator=gen(4)))
    c.q[:, :, 0] = 1.0
    close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets, scale=1.0), *c.reference(scale=1.0))


def test_prompt_values_of_very_different_rows_in_8_bits():
    """Value rows of 2^-60 and of 2^20 side by side, zeros among them; queries of 2^-30 and of 2^30."""
    n = 300
    c = Case([n], [200], heads=4, kv=1, d=64, cache=E4M3)
    g = gen(5)
    v = torch.randn(n, 1, 64, device="cuda", generator=g) * torch.exp2(torch.randint(-60, 20, (n, 1, 1), device="cuda", generator=g).float())
    v[7] = 0
    fill(c, 0, torch.randn(n, 1, 64, device="cuda", generator=g), v)
    close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets), *c.reference())
    fill(c, 0, torch.randn(n, 1, 64, device="cuda", generator=g) * 2.0 ** -30, v)
    c.q = (c.q.float() * 2.0 ** 30).bfloat16()
    close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets), *c.reference())
    fill(c, 0, torch.randn(n, 1, 64, device="cuda", generator=g) * 2.0 ** 30, v)
    c.q = (c.q.float() * 2.0 ** -60).bfloat16()
    close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets), *c.reference())
    close(sw.decode_attention(c.q[-1:], c.cache, c.table, c.lengths), *(x[-1:] for x in c.reference()))


@pytest.mark.parametrize("cache", [None, E4M3])
def test_few_tokens_behind_many_rows_in_parts(cache):
    """Where the cache is cut into parts: tokens that see a part only, windows that leave parts empty, several sequences of very different lengths."""
    for lengths, counts, heads, kv, window in (([5000], [3], 4, 1, 0), ([5000], [70], 8, 2, 0), ([5000, 60, 0, 1300], [2, 60, 0, 5], 2, 1, 0), ([5000], [40], 4, 1, 300), ([4000], [1], 1, 1, 0), ([900], [20], 130, 1, 0)):
        c = Case(lengths, counts, heads=heads, kv=kv, d=80, page=64, dtype=torch.float16, cache=cache, seed=counts[0])
        close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets, window=window), *c.reference(window=window))


def test_prompt_strided_and_misaligned_queries_and_results():
    c = Case([300, 41], [100, 41], heads=6, kv=2, d=80, dtype=torch.float16)
    want, tol = c.reference()
    buffer = torch.zeros(141, 6 * 83 + 5, dtype=torch.float16, device="cuda")
    q = torch.as_strided(buffer, (141, 6, 80), (6 * 83 + 5, 83, 1), 3)
    q.copy_(c.q)
    back = torch.full((141, 6 * 81 + 1), 7.0, dtype=torch.float16, device="cuda")
    out = torch.as_strided(back, (141, 6, 80), (6 * 81 + 1, 81, 1), 1)
    assert sw.prompt_attention(q, c.cache, c.table, c.lengths, c.offsets, out=out) is out
    close(out, want, tol)
    assert bool((back[:, 0] == 7).all())
    close(sw.prompt_attention(c.q.transpose(0, 1).contiguous().transpose(0, 1), c.cache, c.table, c.lengths, c.offsets), want, tol)


def test_rows_outside_every_sequence_stay_and_more_new_tokens_than_rows_give_zeros():
    c = Case([20, 30], [20, 30], heads=4, kv=1)
    want, tol = c.reference()
    q = torch.cat([torch.full((3, 4, 128), math.nan, device="cuda").bfloat16(), c.q, torch.full((5, 4, 128), math.nan, device="cuda").bfloat16()])
    out = torch.full_like(q, 9.0)
    offsets = (c.offsets + 3).to(torch.int32)
    sw.prompt_attention(q, c.cache, c.table, c.lengths, offsets, out=out)
    close(out[3:53], want, tol)
    assert bool((out[:3] == 9).all()) and bool((out[53:] == 9).all())
    # the first sequence has 12 rows for its 20 new tokens
    lengths = torch.tensor([12, 30], dtype=torch.int32, device="cuda")
    out = sw.prompt_attention(c.q, c.cache, c.table, lengths, c.offsets)
    assert not bool(out[:8].any())
    close(out[20:], want[20:], tol[20:])
    # row 8 + i of q is the token at position i
    d = Case([20, 30], [20, 30], heads=4, kv=1)
    d.q = torch.cat([c.q[8:20], c.q[8:20], c.q[20:]])
    d.counts, d.lengths_host, d.offsets_host = [12, 30], [12, 30], [0, 12, 42]
    d.k64[0], d.v64[0] = c.k64[0][:12], c.v64[0][:12]
    d.q = torch.cat([c.q[8:20], c.q[20:]])
    close(out[8:20], *(x[:12] for x in d.reference()))


@pytest.mark.parametrize("cache", [None, E4M3])
@pytest.mark.parametrize("window", [0, 5000])
def test_more_parts_than_fit_the_gpu_at_once(cache, window):
    """Few tokens behind many rows, of so many sequences that their parts are taken in turns."""
    counts = [200 - 7 * i for i in range(24)]
    c = Case([7000 - 211 * i for i in range(23)] + [39], counts, heads=2, kv=2, d=64, page=16, cache=cache)
    close(sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets, window=window), *c.reference(window=window))


@pytest.mark.parametrize("cache", [None, E4M3])
def test_many_more_new_tokens_than_rows_give_zeros(cache):
    """300 new tokens of a sequence that has 12 rows: whole blocks of tokens see nothing."""
    c = Case([300, 40], [300, 40], heads=4, kv=1, cache=cache)
    out = torch.full_like(c.q, 9.0)
    sw.prompt_attention(c.q, c.cache, c.table, torch.tensor([12, 40], dtype=torch.int32, device="cuda"), c.offsets, out=out)
    assert not bool(out[:288].any())
    want, tol = c.reference()
    close(out[300:], want[300:], tol[300:])
    c.q, c.counts, c.lengths_host, c.offsets_host = c.q[288:300], [12], [12], [0, 12]
    c.k64[0], c.v64[0] = c.k64[0][:12], c.v64[0][:12]
    close(out[288:300], *c.reference())


@pytest.mark.parametrize("offsets", [[0, 40, 0, 40, 0, 40, 0, 40, 0], [0, 1, 40, 3, 40, 2, 40, 0, 40], [40] * 9, [0] * 8 + [10 ** 9]])
def test_sequences_that_overlap_touch_nothing_else(offsets):
    """Offsets that go to and fro, where the cache is cut into parts: more blocks of tokens than there are places for."""
    c = Case([3000], [40], heads=1, kv=1, d=64, page=64)
    table, lengths = c.table.expand(8, -1).contiguous(), c.lengths.expand(8).contiguous()
    out = torch.full((40 + 64, 1, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    sw.prompt_attention(c.q, c.cache, table, lengths, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=out[:40])
    torch.cuda.synchronize()
    binding.strassen_device_status()
    assert bool((out[40:] == 9).all())


@pytest.mark.parametrize("offsets", [[0, 90, 30], [-5, 10, 10 ** 9], [2 ** 31 - 1, 0, 5], [-2 ** 31, -7, -1]])
def test_offsets_of_any_kind_touch_nothing_else(offsets):
    c = Case([20, 30], [20, 30], heads=4, kv=1)
    out = torch.full((50 + 64, 4, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    sw.prompt_attention(c.q, c.cache, c.table, c.lengths, torch.tensor(offsets, dtype=torch.int32, device="cuda"), out=out[:50])
    torch.cuda.synchronize()
    binding.strassen_device_status()
    assert bool((out[50:] == 9).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("at", [0, 1, 150, 255, 399])
@pytest.mark.parametrize("cache", [None, E4M3])
def test_what_a_token_does_not_see_has_no_effect(bad, which, at, cache):
    """One bad row at a position of a prompt: the tokens before it, and those a window later, are as if it were finite; the others are not."""
    window = 70
    c = Case([400], [400], heads=4, kv=2, d=64, page=16, cache=cache)
    for w in (0, window):
        want, tol = c.reference(window=w)
        store = c.cache.k if which == "k" else c.cache.v
        page, slot = int(c.table[0, at // 16]), at % 16
        if cache == E4M3:                                        # there an infinity can be a row's scale
            store, column = c.cache.k_scale if which == "k" else c.cache.v_scale, ()
        else:
            column = (5,)
        keep = store[page, 1, slot].clone()
        store[(page, 1, slot) + column] = bad
        got = sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets, window=w)
        one = sw.decode_attention(c.q[-1:], c.cache, c.table, c.lengths, window=w)
        store[page, 1, slot] = keep
        sees = torch.zeros(400, dtype=torch.bool, device="cuda")
        sees[at:at + w if w else None] = True
        close(got[~sees], want[~sees], tol[~sees])
        close(got[:, :2], want[:, :2], tol[:, :2])
        if cache == E4M3:
            assert not bool(torch.isfinite(got[sees][:, 2:]).any()) if which == "v" else (bad == bad or bool(torch.isnan(got[sees][:, 2:]).all()))
        elif which == "v":                                       # the column is what the definition gives, the others are as ever
            assert bool((got[sees][:, 2:, 5].float().nan_to_num(1.5, 2.5, -2.5) == torch.tensor(bad).nan_to_num(1.5, 2.5, -2.5).item()).all())
            others = [i for i in range(64) if i != 5]
            close(got[..., others], want[..., others], tol[..., others])
        elif bad != bad:
            assert bool(torch.isnan(got[sees][:, 2:]).all())
        if not bool(sees[-1]):
            close(one, want[-1:], tol[-1:])


@pytest.mark.parametrize("cache", [None, E4M3])
@pytest.mark.parametrize("heads,kv,d", [(8, 8, 64), (8, 2, 128), (32, 2, 80), (12, 1, 128)])
@pytest.mark.parametrize("lengths", [[65, 0, 300, 1], [2000], [1000, 640, 641, 37, 999], [5000], [500 - 11 * i for i in range(40)]], ids=lambda x: "%dx%d" % (len(x), max(x)))
def test_few_short_sequences_in_narrow_and_wide_tables(lengths, heads, kv, d, cache):
    """A table's width says what there may be to do, the lengths what there is: work is cut by the first, results go by the second."""
    c = Case(lengths, heads=heads, kv=kv, d=d, page=16, dtype=torch.float16 if d == 80 else torch.bfloat16, cache=cache, seed=5)
    for window in (0, 130):
        want, tol = c.reference(window=window)
        for rows in (0, 1500, 7000, 40000, 200000):
            table = torch.nn.functional.pad(c.table, (0, rows // c.page), value=-1)
            out = torch.full_like(c.q, 9.0)
            close(sw.decode_attention(c.q, c.cache, table, c.lengths, window=window, out=out), want, tol)
            assert torch.equal(out, sw.decode_attention(c.q, c.cache, table, c.lengths, window=window))


@pytest.mark.parametrize("cache", [None, E4M3])
def test_bad_queries_of_one_token_stay_with_their_heads(cache):
    c = Case([300, 41, 700], heads=8, kv=2, cache=cache)
    want, tol = c.reference()
    c.q[1, 3, 3] = math.nan
    c.q[2, 6, 3] = math.inf
    got = sw.decode_attention(c.q, c.cache, c.table, c.lengths)
    good = torch.ones(3, 8, dtype=torch.bool, device="cuda")
    good[1, 3] = good[2, 6] = False
    close(got[good], want[good], tol[good])
    assert bool(torch.isnan(got[1, 3]).all())


@pytest.mark.parametrize("cache_type", [torch.bfloat16, E4M3])
def test_pages_beyond_four_gigabytes(cache_type):
    """The last pages of a cache whose offsets in elements, and in bytes, take more than 32 bits."""
    kv, d, page = 4, 128, 128
    pages = (2 ** 32 + 2 ** 29) // (kv * d * page)
    cache = sw.PagedCache.empty(pages, kv, d, page, cache_type)
    f = frequencies(d)
    g = gen(21)
    n = 200
    k, v, q = (torch.randn(n, h, d, device="cuda", generator=g).bfloat16() for h in (kv, kv, 8))
    lengths, offsets = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([n], [0, n]))
    small = sw.PagedCache.empty(2, kv, d, page, cache_type)
    got = []
    for c, table in ((cache, [[pages - 1, pages - 2]]), (small, [[0, 1]])):
        table = torch.tensor(table, dtype=torch.int32, device="cuda")
        turned = sw.rotate_append(q, k, v, c, table, lengths, f, offsets)
        got.append((turned, sw.prompt_attention(turned, c, table, lengths, offsets), sw.decode_attention(turned[-1:], c, table, lengths)))
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_a_cache_without_pages():
    c = Case([30], [5], heads=4, kv=1, d=64)
    for dtype in (torch.bfloat16, E4M3):
        cache = sw.PagedCache.empty(0, 1, 64, 16, dtype)
        sw.rotate_append(c.q, c.q[:, :1], c.q[:, :1], cache, c.table, c.lengths, None, c.offsets)
        assert not bool(sw.prompt_attention(c.q, cache, c.table, c.lengths, c.offsets).any())
        assert not bool(sw.decode_attention(c.q[:1], cache, c.table, c.lengths).any())


def test_bad_queries_stay_in_their_rows():
    c = Case([300, 41], [300, 41], heads=4, kv=2)
    want, tol = c.reference()
    c.q[77, 1, 3] = math.nan
    c.q[310, 2, 3] = math.inf
    got = sw.prompt_attention(c.q, c.cache, c.table, c.lengths, c.offsets)
    good = torch.ones(341, 4, dtype=torch.bool, device="cuda")
    good[77, 1] = good[310, 2] = False
    close(got[good], want[good], tol[good])
    assert bool(torch.isnan(got[77, 1]).all())


# ---- storing -----------------------------------------------------------------------------------------------------------

def turned(x, positions, frequencies, interleaved):
    """x (tokens, heads, d) in 64 bits, turned."""
    x, r = x.double().clone(), 2 * frequencies.shape[0]
    a = positions.double()[:, None, None] * frequencies.double()
    first, second = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    new = first * a.cos() - second * a.sin(), first * a.sin() + second * a.cos()
    if interleaved:
        x[..., 0:r:2], x[..., 1:r:2] = new
    else:
        x[..., :r // 2], x[..., r // 2:r] = new
    return x


def frequencies(r):
    return (500000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)).float().cuda()


def check_append(heads, kv, d, dtype, cache_type, rotary, interleaved, lengths, counts, page=16, layout="pages", offset=0, in_place=False, single=False):
    g = gen(heads * d + rotary)
    tokens, batch = sum(counts), len(lengths)
    width = max(1, max(-(-n // page) for n in lengths))
    pages = batch * width + 1
    table = torch.randperm(pages, device="cuda", generator=g)[:batch * width].view(batch, width).to(torch.int32)
    shape = {"pages": (pages, kv, page, d), "rows": (pages, page, kv, d)}[layout]
    k, v = (torch.full(shape, 3.0, device="cuda").to(cache_type) for _ in range(2))
    if layout == "rows":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    scales = [torch.full((pages, kv, page), 3.0, device="cuda") if cache_type == E4M3 else None for _ in range(2)]
    cache = sw.PagedCache(k, v, *scales)
    wide = (heads + 2 * kv) * d
    qkv = torch.randn(tokens * (wide + offset) + offset, device="cuda", generator=g).to(dtype)
    rows = torch.as_strided(qkv, (tokens, heads + 2 * kv, d), (wide + offset, d, 1), offset)
    q, nk, nv = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
    positions = torch.cat([torch.arange(n - m, n) for n, m in zip(lengths, counts)]).cuda()
    owner = torch.cat([torch.full((m,), b) for b, m in enumerate(counts)]).cuda()
    f = frequencies(rotary) if rotary else None
    want_q, want_k, want_v = q.double().clone(), nk.double().clone(), nv.double().clone()
    if rotary:
        want_q, want_k = turned(q, positions, f, interleaved), turned(nk, positions, f, interleaved)
    offsets = torch.tensor([sum(counts[:i]) for i in range(batch + 1)], dtype=torch.int32, device="cuda")
    keep = qkv.clone()
    got = sw.rotate_append(q, nk, nv, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), f, None if single else offsets, interleaved, out=q if in_place else None)
    u = HALF_STEP[dtype]
    # the angle's cosine and sine are within 2^-22 (a fraction of a turn in 32 bits, and their own rounding), products and sum 3 roundings in 32 bits
    size = want_q.abs().amax() * 2.0 ** -20
    close(got, want_q, u * want_q.abs() + size + 2.0 ** -25 * (dtype == torch.float16))
    if in_place:
        assert got is q
        keep = torch.as_strided(keep, (tokens, heads + 2 * kv, d), (wide + offset, d, 1), offset)
        assert torch.equal(keep[:, heads:], rows[:, heads:])
    else:
        assert torch.equal(keep, qkv)
    at = table[owner, positions // page].long(), positions % page
    touched = torch.zeros(pages, kv, page, dtype=torch.bool, device="cuda")
    touched[at[0], :, at[1]] = True
    for store, scale, want in ((cache.k, cache.k_scale, want_k), (cache.v, cache.v_scale, want_v)):
        have = store[at[0], :, at[1]] if cache_type != E4M3 else store.view(torch.uint8)[at[0], :, at[1]].view(E4M3)
        if cache_type == E4M3:
            s = (want.abs().amax(-1) / 448).clamp_min(2.0 ** -64)
            have_s = scale[at[0], :, at[1]].double()
            assert bool(((have_s - s).abs() <= s * 2.0 ** -18).all())
            # half a step of e4m3 (at most 16 of 448), 2^-10 where it is subnormal, and the row's own errors above
            tol = (want.abs() * 2.0 ** -4).clamp_min(2.0 ** -10 * s[..., None]) + s[..., None] * 448 * 2.0 ** -17
            close(have.double() * have_s[..., None], want, tol)
            assert bool((scale[~touched] == 3).all())
        else:
            close(have, want, u * want.abs() + size + 2.0 ** -25 * (dtype == torch.float16))
        assert bool((store.float()[~touched] == 3).all())


@pytest.mark.parametrize("dtype,cache", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, E4M3), (torch.float16, E4M3)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("heads,kv,d,rotary", [(32, 8, 128, 128), (12, 12, 80, 64), (4, 2, 96, 96), (2, 1, 112, 20), (1, 1, 64, 2), (3, 1, 16, 0), (5, 5, 48, 48), (7, 1, 128, 36)])
def test_append(heads, kv, d, rotary, interleaved, dtype, cache):
    check_append(heads, kv, d, dtype, cache, rotary, interleaved, [37, 100, 0, 1], [37, 9, 0, 1])


@pytest.mark.parametrize("cache", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("d", [16, 32, 48, 64, 80, 96, 112, 128])
def test_append_many_tokens_of_few_heads(d, cache):
    """Blocks of up to 64 tokens, of several sequences, and rows of 1 to 8 lanes."""
    check_append(1, 1, d, torch.bfloat16, cache, d if d % 32 else 32, d % 32 == 0, [12000, 700, 0, 65, 9001, 3000, 64], [12000, 3, 0, 65, 9001, 2999, 64], page=32)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("cache", [torch.bfloat16, E4M3])
def test_append_one_token_each(cache, in_place):
    check_append(32, 8, 128, torch.bfloat16, cache, 128, False, [700, 1, 33, 64, 65], [1] * 5, in_place=in_place, single=True)


@pytest.mark.parametrize("interleaved", [False, True])
def test_append_in_place_many_and_other_orders(interleaved):
    check_append(12, 4, 80, torch.float16, torch.float16, 64, interleaved, [400, 1000], [400, 333], in_place=True, layout="rows", page=64)
    check_append(12, 4, 80, torch.float16, E4M3, 64, interleaved, [400, 1000], [400, 333], in_place=True, layout="rows", page=64)


@pytest.mark.parametrize("offset", [1, 2, 4, 5])
@pytest.mark.parametrize("cache", [torch.float16, E4M3])
def test_append_misaligned(offset, cache):
    check_append(6, 2, 80, torch.float16, cache, 80, False, [50, 20], [50, 3], offset=offset)
    check_append(6, 2, 80, torch.float16, cache, 40, True, [50, 20], [50, 3], offset=offset, in_place=True)


def test_append_far_positions():
    """Angles of positions whose product with a frequency has no fraction left in 32 bits."""
    d, page = 64, 1024
    start = 2 ** 24 + 12345
    f = frequencies(d)
    width = start // page + 1
    cache = sw.PagedCache(*(torch.zeros(2, 1, page, d, device="cuda") .bfloat16() for _ in range(2)))
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    q, k, v = (torch.randn(1, 1, d, device="cuda", generator=gen(i)).bfloat16() for i in range(3))
    got = sw.rotate_append(q, k, v, cache, table, torch.tensor([start + 1], dtype=torch.int32, device="cuda"), f)
    want = turned(q, torch.tensor([start], device="cuda"), f, False)
    close(got, want, want.abs() * 2.0 ** -8 + 2.0 ** -18)
    want = turned(k, torch.tensor([start], device="cuda"), f, False)
    close(cache.k[1, :, start % page], want[0], want[0].abs() * 2.0 ** -8 + 2.0 ** -18)


def test_append_leaves_out_what_has_no_place():
    d, page = 64, 16
    k = torch.randn(30, 2, d, device="cuda", generator=gen(1)).bfloat16()
    cache = sw.PagedCache(*(torch.full((4, 2, page, d), 3.0, device="cuda").bfloat16() for _ in range(2)))
    q = k.clone()
    out = torch.full_like(q, 9.0)
    # tokens 0..9: pages that are not there; 10..19: two of them before the sequence's first row; 20..24 behind the table; 25..29 of no sequence
    table = torch.tensor([[4, -1], [2, 3], [-7, 1]], dtype=torch.int32, device="cuda")
    offsets = torch.tensor([0, 10, 20, 25], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([20, 8, 37], dtype=torch.int32, device="cuda")
    sw.rotate_append(q, k, k, cache, table, lengths, None, offsets, out=out)
    want = torch.full((4, 2, page, d), 3.0, device="cuda").bfloat16()
    want[2, :, :8] = k[12:20].transpose(0, 1)
    assert torch.equal(cache.k, want) and torch.equal(cache.v, want)
    assert torch.equal(out[12:25], q[12:25]) and torch.equal(out[:10], q[:10]) and bool((out[10:12] == 9).all()) and bool((out[25:] == 9).all())
    for bad in ([-5, 3, 2, 10 ** 9], [2 ** 31 - 1, -2 ** 31, 5, 6], [30, 20, 10, 0]):
        sw.rotate_append(q, k, k, cache, table, lengths, None, torch.tensor(bad, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()


def test_append_bad_values_in_8_bits():
    """A row with NaN is NaN throughout, and its neighbours are not touched by it."""
    cache = sw.PagedCache.empty(2, 2, 64, 16, E4M3)
    k = torch.randn(4, 2, 64, device="cuda", generator=gen(1)).bfloat16()
    k[1, 0, 7] = math.nan
    k[3, 1] = 0
    table, lengths, offsets = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([[1]], [4], [0, 4]))
    sw.rotate_append(None, k, k, cache, table, lengths, None, offsets)
    rows = cache.k.float()[1] * cache.k_scale[1][..., None]
    assert bool(torch.isnan(rows[0, 1]).all()) and bool(torch.isnan(cache.k_scale[1, 0, 1]))
    assert bool(torch.isfinite(rows[0, [0, 2, 3]]).all()) and bool(torch.isfinite(rows[1, :4]).all())
    assert not bool(rows[1, 3].any()) and float(cache.k_scale[1, 1, 3]) == 2.0 ** -64


# ---- together ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("cache_type", [torch.bfloat16, E4M3])
def test_a_prompt_in_parts_and_token_by_token_is_the_prompt_at_once(cache_type):
    """Stored and attended in parts of 50, 1, 1 and 28 tokens, and all at once: the same rows of the cache, results within twice the tolerance."""
    c = Case([80], [80], heads=8, kv=2, d=64, page=16)
    f = frequencies(64)
    g = gen(9)
    k, v = (torch.randn(80, 2, 64, device="cuda", generator=g).bfloat16() for _ in range(2))
    caches = [sw.PagedCache.empty(8, 2, 64, 16, cache_type) for _ in range(2)]
    for x in caches:
        x.k.view(torch.uint8).zero_(), x.v.view(torch.uint8).zero_()
    table = torch.randperm(8, device="cuda", generator=g)[None, :5].to(torch.int32)
    done, parts = 0, []
    for n in (50, 1, 1, 28):
        rows = slice(done, done + n)
        done += n
        lengths, offsets = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([done], [0, n]))
        q = sw.rotate_append(c.q[rows], k[rows], v[rows], caches[0], table, lengths, f, offsets if n > 1 else None)
        parts.append(sw.prompt_attention(q, caches[0], table, lengths, offsets) if n > 1 else sw.decode_attention(q, caches[0], table, lengths))
    q = sw.rotate_append(c.q, k, v, caches[1], table, c.lengths, f, c.offsets)
    whole = sw.prompt_attention(q, caches[1], table, c.lengths, c.offsets)
    used = table[0].long()
    assert torch.equal(caches[0].k.view(torch.uint8)[used], caches[1].k.view(torch.uint8)[used]) and torch.equal(caches[0].v.view(torch.uint8)[used], caches[1].v.view(torch.uint8)[used])
    c.q = q
    for i, store, scales in ((0, caches[1].k, caches[1].k_scale), (1, caches[1].v, caches[1].v_scale)):
        x = store.double()[used] * (scales.double()[used][..., None] if scales is not None else 1)
        (c.k64, c.v64)[i][0] = x.transpose(0, 1).flatten(1, 2).transpose(0, 1)
    want, tol = c.reference()
    close(whole, want, tol)
    close(torch.cat(parts), want, tol)


def block(width, heads, kv, d, g, dtype=torch.bfloat16, **kw):
    from paper_1202_3173_b200.feed_forward import quantize_w4
    weights, plain = [], []
    for n, k in (((heads + 2 * kv) * d, width), (width, heads * d)):
        q, s, z = quantize_w4(torch.randn(n, k, device="cuda", generator=g) * k ** -0.5, 64)
        weights.append(sw.W4Matrix(q, s, z, k=k, group=64))
        nibbles = torch.stack([q & 15, q >> 4], -1).view(n, k).double()
        plain.append(s.double().repeat_interleave(64, 1)[:, :k] * (nibbles - z.double().repeat_interleave(64, 1)[:, :k]))
    norm = (1 + 0.1 * torch.randn(width, device="cuda", generator=g)).to(dtype)
    return sw.SelfAttention(norm, *weights, heads, **kw), plain


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("cache_type", ["16 bits", E4M3])
def test_the_block(dtype, cache_type):
    """The block is the operators one after another: bit for bit, for a prompt of two sequences and for a token each."""
    width, heads, kv, d = 256, 6, 2, 64
    f = frequencies(32)
    blk, _ = block(width, heads, kv, d, gen(2), dtype, frequencies=f, window=40)
    half = dtype if dtype != torch.float32 else torch.bfloat16
    cache_type = half if cache_type == "16 bits" else cache_type
    caches = [sw.PagedCache.empty(8, kv, d, 16, cache_type) for _ in range(2)]
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    x, r = (torch.randn(72, width, device="cuda", generator=gen(3)).to(dtype) for _ in range(2))
    for rows, lengths, offsets in ((slice(0, 70), [30, 40], [0, 30, 70]), (slice(70, 72), [31, 41], None)):
        lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        offsets = torch.tensor(offsets, dtype=torch.int32, device="cuda") if offsets else None
        y, h = blk(x[rows], r[rows], caches[0], table, lengths, offsets)
        assert y.dtype == dtype and h.dtype == dtype
        n, s, want_h = sw.rms_norm_quant(x[rows], blk.norm_weight, residual=r[rows])
        qkv = blk.qkv(n, s, dtype=half).view(-1, heads + 2 * kv, d)
        q = sw.rotate_append(qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:], caches[1], table, lengths, f, offsets)
        a = sw.prompt_attention(q, caches[1], table, lengths, offsets, window=40) if offsets is not None else sw.decode_attention(q, caches[1], table, lengths, window=40)
        assert torch.equal(h, want_h) and torch.equal(y, blk.o(a.flatten(1)).to(dtype))


def test_the_block_without_rows():
    blk, _ = block(256, 6, 2, 64, gen(2))
    cache = sw.PagedCache.empty(8, 2, 64, 16)
    x = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")
    y, h = blk(x, x, cache, torch.empty(0, 4, dtype=torch.int32, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"))
    assert y.shape == h.shape == (0, 256)


def test_the_example_runs():
    from paper_1202_3173_b200 import attention
    attention.main()


@pytest.mark.parametrize("cache", [None, E4M3])
def test_same_bits_again_and_in_a_graph_replayed_for_other_lengths(cache):
    c = Case([500, 1200, 64], [1, 1, 1], heads=8, kv=2, cache=cache, seed=1)
    p = Case([500, 1200, 64], [300, 40, 64], heads=8, kv=2, cache=cache, seed=1)
    shorter = torch.tensor([499, 700, 33], dtype=torch.int32, device="cuda")
    first = [sw.decode_attention(c.q, c.cache, c.table, n) for n in (c.lengths, shorter)]
    first_p = [sw.prompt_attention(p.q, p.cache, p.table, n, p.offsets) for n in (p.lengths, shorter)]
    for _ in range(3):
        assert torch.equal(first[0], sw.decode_attention(c.q, c.cache, c.table, c.lengths))
        assert torch.equal(first_p[0], sw.prompt_attention(p.q, p.cache, p.table, p.lengths, p.offsets))
    lengths = c.lengths.clone()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graphs, outs = [], []
        for call in (lambda: sw.decode_attention(c.q, c.cache, c.table, lengths), lambda: sw.prompt_attention(p.q, p.cache, p.table, lengths, p.offsets)):
            call()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                outs.append(call())
            graphs.append(graph)
    for i, n in enumerate((c.lengths, shorter, c.lengths)):
        lengths.copy_(n)
        torch.cuda.synchronize()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], first[i % 2]) and torch.equal(outs[1], first_p[i % 2])


def test_calls_on_two_streams_at_once():
    c = [Case([3000 + i, 200], heads=8, kv=2, seed=i) for i in range(2)]
    want = [sw.decode_attention(x.q, x.cache, x.table, x.lengths) for x in c]
    p = [Case([900 + i, 200], [900 + i, 100], heads=8, kv=2, seed=i) for i in range(2)]
    want_p = [sw.prompt_attention(x.q, x.cache, x.table, x.lengths, x.offsets) for x in p]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got, got_p = [[], []], [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(sw.decode_attention(c[i].q, c[i].cache, c[i].table, c[i].lengths))
                got_p[i].append(sw.prompt_attention(p[i].q, p[i].cache, p[i].table, p[i].lengths, p[i].offsets))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i]) and all(torch.equal(x, want_p[i]) for x in got_p[i])


def test_a_captured_step_of_generation_follows_the_lengths():
    """Store, attend and count up in one graph, replayed: what calls one after another give."""
    heads, kv, d, steps = 8, 2, 128, 40
    g = gen(11)
    f = frequencies(d)
    rows = torch.randn(steps, 2, heads + 2 * kv, d, device="cuda", generator=g).bfloat16()
    def run(graphed):
        cache = sw.PagedCache.empty(10, kv, d, 16)
        cache.k.zero_(), cache.v.zero_()
        table = torch.arange(10, dtype=torch.int32, device="cuda").view(2, 5)
        lengths = torch.tensor([0, 23], dtype=torch.int32, device="cuda")
        x, out, outs = torch.zeros_like(rows[0]), torch.zeros(2, heads, d, device="cuda").bfloat16(), []
        def step():
            lengths.add_(1)
            q = sw.rotate_append(x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:], cache, table, lengths, f)
            sw.decode_attention(q, cache, table, lengths, out=out)
        if graphed:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                step()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    step()
            torch.cuda.synchronize()
            cache.k.zero_(), cache.v.zero_()
            lengths.copy_(torch.tensor([0, 23], dtype=torch.int32))
        for i in range(steps):
            x.copy_(rows[i])
            if graphed:
                graph.replay()
            else:
                step()
            outs.append(out.clone())
        return torch.stack(outs), cache.k.clone()
    a, b = run(False), run(True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- refusals that need a device -------------------------------------------------------------------------------------------

def test_refusals():
    c = Case([30, 20], [1, 1], heads=4, kv=2, d=64)
    p = Case([30, 20], [10, 20], heads=4, kv=2, d=64)
    f = frequencies(64)
    k = p.q[:, :2].contiguous()
    decode = lambda **x: sw.decode_attention(**{**dict(q=c.q, cache=c.cache, table=c.table, lengths=c.lengths), **x})
    prompt = lambda **x: sw.prompt_attention(**{**dict(q=p.q, cache=p.cache, table=p.table, lengths=p.lengths, offsets=p.offsets), **x})
    append = lambda **x: sw.rotate_append(**{**dict(q=p.q, k=k, v=k, cache=p.cache, table=p.table, lengths=p.lengths, frequencies=f, offsets=p.offsets), **x})
    for call in (decode, prompt, append):
        call()
    for call, change in (
            (decode, dict(q=c.q.half())), (decode, dict(q=c.q.float())), (decode, dict(q=c.q[:1])), (decode, dict(q=c.q[..., :32])), (decode, dict(q=c.q[0])), (decode, dict(q=c.q.cpu())),
            (decode, dict(q=c.q.transpose(1, 2).contiguous().transpose(1, 2))), (decode, dict(table=c.table.long())), (decode, dict(table=c.table[:1])), (decode, dict(table=c.table.cpu())),
            (decode, dict(table=c.table.t().contiguous().t())), (decode, dict(lengths=c.lengths.long())), (decode, dict(lengths=c.lengths.cpu())), (decode, dict(lengths=c.lengths[:, None])),
            (decode, dict(out=torch.empty_like(c.q).half())), (decode, dict(out=torch.empty_like(c.q)[:1])), (decode, dict(q=c.q.clone().requires_grad_())),
            (prompt, dict(offsets=None)), (prompt, dict(offsets=p.offsets.long())), (prompt, dict(offsets=p.offsets[:2])), (prompt, dict(offsets=p.offsets.cpu())),
            (append, dict(k=k.half())), (append, dict(v=k[:, :1])), (append, dict(k=k[:5])), (append, dict(frequencies=f.double())), (append, dict(frequencies=frequencies(66))),
            (append, dict(frequencies=f[:0])), (append, dict(frequencies=f.cpu())), (append, dict(offsets=None)), (append, dict(q=None, out=p.q)), (append, dict(k=k.clone().requires_grad_())),
            (append, dict(out=torch.empty_like(p.q)[:, :2]))):
        with pytest.raises(ValueError):
            call(**change)
    for call, change in ((decode, dict(q=c.q[:, :3].contiguous())), (decode, dict(window=-1)), (decode, dict(scale=math.nan)), (decode, dict(scale=math.inf)), (decode, dict(out=c.q)),
                         (prompt, dict(out=p.q)), (prompt, dict(window=-5)), (append, dict(out=torch.empty(30, 8, 64, device="cuda").bfloat16()[:, ::2], q=p.q))):
        if call is append:
            call(**change)                  # other strides are fine
            continue
        with pytest.raises(StrassenError):
            call(**change)
    with torch.no_grad():
        decode(q=c.q.clone().requires_grad_())
    before = c.q._version
    out = torch.empty_like(c.q)
    version = out._version
    decode(out=out)
    assert out._version > version and c.q._version == before
    version = p.cache.k._version
    append()
    assert p.cache.k._version > version


def test_cache_refusals():
    k = torch.zeros(4, 2, 16, 64, device="cuda").bfloat16()
    sw.PagedCache(k, k.clone())
    eight = k.to(E4M3)
    scale = torch.zeros(4, 2, 16, device="cuda")
    sw.PagedCache(eight, eight.clone(), scale, scale.clone())
    for args in ((k.float(), k.float()), (k.cpu(), k.cpu()), (k[0], k[0]), (k, k[:2]), (k, k.half()), (k, k.transpose(1, 2).contiguous().transpose(1, 2)), (k, k, scale, scale), (eight, eight),
                 (eight, eight, scale[:2], scale), (eight, eight, scale.half(), scale), (k[:, :, :12], k[:, :, :12]), (k[..., ::2], k[..., ::2]), (k[..., :60], k[..., :60]), (k[..., 4:36], k[..., 4:36]),
                 (eight[..., :8], eight[..., :8], scale, scale), (k[:, :1, :1].expand(4, 2, 16, 64), k[:, :1, :1].expand(4, 2, 16, 64)),
                 (torch.zeros(1, 1, 16, 136, device="cuda").bfloat16(), torch.zeros(1, 1, 16, 136, device="cuda").bfloat16())):
        with pytest.raises(ValueError):
            sw.PagedCache(*args)
