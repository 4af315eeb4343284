"""Every row that a token sees counts once, and no other: attention with values of one row at a time.

Random values cannot show it: over 40000 of them a result is so small beside the bound on its error that a lost step of rows stays within it.  So here column c of key head h holds
nothing but one row's value, a power of two, and the result in that column is that row's weight.  A few launches have every row in some column.  Scores are 0, or rise and fall in steps
along the sequence, so that parts of it have maxima of their own.

Tolerance: the weight is rounded once to 16 bits and the result once, u each (half a step of the type); scores are exact, their exponentials and the sums of up to 2^17 terms in
32 bits 2^-17; a result that f16 holds without all its bits, 2^-25.  A row lost is 1 of 1, one counted twice the same.
"""
import math

import pytest
import torch

import paper_1202_3173_b200 as sw

E4M3 = torch.float8_e4m3fn
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def weights(n, steps, device):
    """Scores of the rows and their weights before they are divided by their sum."""
    j = torch.arange(n, device=device)
    score = (j // 61 % 9).double() / 2 if steps else torch.zeros(n, dtype=torch.float64, device=device)
    return score, score.exp()


def expected(n, count, w, first, kv, group, d, value, window):
    """(count, kv * group, d): what the tokens at positions n - count .. n - 1 get when row first + h * d + c is in column c of key head h."""
    device = w.device
    p = torch.arange(n - count, n, device=device)[:, None]
    j = torch.arange(kv * d, device=device)[None] + first
    seen = (j <= p) & (j < n) & ((j > p - window) if window else True)
    total = torch.cat([torch.zeros(1, dtype=torch.float64, device=device), w.cumsum(0)])
    low = (p - window + 1).clamp_min(0) if window else torch.zeros_like(p)
    out = torch.where(seen, w[j.clamp_max(n - 1)], torch.zeros_like(w[:1])) * value / (total[p + 1] - total[low])
    return out.view(count, kv, 1, d).expand(count, kv, group, d).reshape(count, kv * group, d)


def check(got, want, dtype):
    tol = want * (2 * HALF_STEP[dtype] + 2.0 ** -17) + (2.0 ** -25 if dtype == torch.float16 else 0.0)
    wrong = ((got.double() - want).abs() > tol) | ~torch.isfinite(got)
    assert not bool(wrong.any()), "%d numbers, the first at %s: %g, not %g" % (int(wrong.sum()), wrong.nonzero()[0].tolist(), float(got[wrong][0]), float(want[wrong][0]))


@pytest.mark.parametrize("steps", [False, True])
def test_the_check_sees_a_row_lost_or_doubled(steps):
    """The mistake is in what is checked, on the CPU: each row of 40000, and a step of 64 at a time."""
    n, d = 40000, 128
    w = weights(n, steps, "cpu")[1]
    for first in (0, 12800, 39936):
        want = expected(n, 1, w, first, 1, 1, d, 2.0 ** 15, 0)
        check(want.to(torch.bfloat16), want, torch.bfloat16)
        for rows in (slice(0, 1), slice(63, 64), slice(0, 64)):
            for factor in (0.0, 2.0):
                bad = want.clone()
                bad[..., rows] *= factor
                with pytest.raises(AssertionError):
                    check(bad.to(torch.bfloat16), want, torch.bfloat16)


class Rows:
    """Sequences in scattered pages, and their caches with the values of some rows only."""

    def __init__(self, lengths, counts, heads, kv, d, page, dtype, cache, steps, extra=0):
        g = torch.Generator("cuda").manual_seed(len(lengths) + d)
        self.lengths_host, self.counts, self.heads, self.kv, self.d, self.page, self.dtype, self.type = lengths, counts, heads, kv, d, page, dtype, cache
        needed = [-(-n // page) for n in lengths]
        pages = sum(needed) + 2
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
        self.table = torch.full((len(lengths), max(needed) + -(-extra // page)), -1, dtype=torch.int32, device="cuda")
        at, places = 0, []
        for b, n in enumerate(needed):
            self.table[b, :n] = order[at:at + n]
            row = torch.arange(lengths[b], device="cuda")
            places.append((self.table[b, row // page].long(), row % page))
            at += n
        self.places = places
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        offsets = [0]
        for n in counts:
            offsets.append(offsets[-1] + n)
        self.offsets_host, self.offsets = offsets, torch.tensor(offsets, dtype=torch.int32, device="cuda")
        k = torch.zeros(pages, kv, page, d, device="cuda").to(cache)
        v = torch.zeros(pages, kv, page, d, device="cuda").to(cache)
        scales = [torch.ones(pages, kv, page, device="cuda") if cache == E4M3 else None for _ in range(2)]
        self.w = []
        for n, (p, s) in zip(lengths, places):
            score, w = weights(n, steps, "cuda")
            store = k.view(torch.uint8) if cache == E4M3 else k
            row = (2 * score)[:, None].expand(n, kv).to(cache)
            store[p, :, s, 0] = row.view(torch.uint8) if cache == E4M3 else row
            self.w.append(w)
        self.cache = sw.PagedCache(k, v, *scales)
        self.v = v.view(torch.uint8) if cache == E4M3 else v
        self.q = torch.zeros(offsets[-1], heads, d, dtype=dtype, device="cuda")
        self.q[..., 0] = 0.5
        self.value = 256.0 if cache == E4M3 else 2.0 ** 15

    def run(self, call, window):
        """`call` with each row in some column."""
        width = self.kv * self.d
        one = torch.tensor(self.value).to(self.type).cuda()
        one = one.view(torch.uint8) if self.type == E4M3 else one
        for first in range(0, max(self.lengths_host), width):
            self.v.zero_()
            for n, (p, s) in zip(self.lengths_host, self.places):
                j = torch.arange(first, max(first, min(n, first + width)), device="cuda")
                if j.numel():
                    self.v[p[j], (j - first) // self.d, s[j], (j - first) % self.d] = one
            got = call(window)
            for b, (n, m) in enumerate(zip(self.lengths_host, self.counts)):
                if m:
                    check(got[self.offsets_host[b]:self.offsets_host[b + 1]], expected(n, m, self.w[b], first, self.kv, self.heads // self.kv, self.d, self.value, window), self.dtype)

    def decode(self, window):
        return sw.decode_attention(self.q, self.cache, self.table, self.lengths, scale=1.0, window=window)

    def prompt(self, window):
        return sw.prompt_attention(self.q, self.cache, self.table, self.lengths, self.offsets, scale=1.0, window=window)


TYPES = [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, E4M3)]


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [False, True])
@pytest.mark.parametrize("dtype,cache", TYPES, ids=["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("lengths,heads,kv,d,page,window", [
    ([40000], 4, 1, 128, 64, 0),                                  # parts by item
    ([30000, 5, 20000], 8, 2, 128, 64, 0), ([25000], 16, 1, 64, 16, 9999), ([30000], 20, 1, 128, 128, 0),
    ([5000 - 97 * i for i in range(40)], 4, 4, 64, 32, 0),        # parts by run
    ([3000 - 61 * i for i in range(45)], 24, 8, 80, 16, 1111),
    ([1000], 32, 8, 128, 64, 0), ([4000], 16, 8, 128, 16, 0), ([1000, 17, 640], 8, 2, 96, 16, 333),        # clusters
    ([900 - 40 * i for i in range(20)], 12, 3, 64, 32, 0),
    ([1 + 37 * i % 700 for i in range(200)], 8, 2, 128, 64, 0)], ids=lambda x: "%dx%d" % (len(x), max(x)) if isinstance(x, list) else str(x))
def test_decode_counts_every_row_once(lengths, heads, kv, d, page, window, dtype, cache, steps):
    r = Rows(lengths, [1] * len(lengths), heads, kv, d, page, dtype, cache, steps)
    r.run(r.decode, window)


@pytest.mark.gpu
@pytest.mark.parametrize("steps", [False, True])
@pytest.mark.parametrize("dtype,cache", TYPES, ids=["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("lengths,counts,heads,kv,d,page,window", [
    ([20000], [100], 8, 2, 128, 64, 0), ([20000], [3], 4, 1, 64, 16, 0), ([15000], [64], 4, 2, 80, 128, 9000),        # parts
    ([5000, 60, 1300], [2, 60, 5], 4, 2, 128, 16, 0), ([7000 - 211 * i for i in range(24)], [200 - 7 * i for i in range(24)], 2, 2, 64, 16, 0),
    ([3000], [3000], 4, 1, 128, 64, 0), ([2500, 1, 130, 700], [2500, 1, 100, 700], 6, 2, 80, 16, 0),
    ([2500], [1200], 4, 1, 64, 32, 300), ([300 + i for i in range(33)], [1 + 5 * i for i in range(33)], 4, 1, 128, 64, 0)], ids=lambda x: "%dx%d" % (len(x), max(x)) if isinstance(x, list) else str(x))
def test_prompts_count_every_row_once(lengths, counts, heads, kv, d, page, window, dtype, cache, steps):
    r = Rows(lengths, counts, heads, kv, d, page, dtype, cache, steps)
    r.run(r.prompt, window)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,cache", TYPES, ids=["bf16", "f16", "e4m3"])
@pytest.mark.parametrize("lengths,counts,heads,kv", [([2048], [2048], 8, 2), ([512], [512], 32, 8), ([512, 70, 1, 300], [64, 70, 1, 8], 4, 2), ([129], [129], 4, 4)], ids=lambda x: "x".join(map(str, x)) if isinstance(x, list) else str(x))
@pytest.mark.parametrize("extra", [0, 6144, 32768, 131072])
def test_prompts_in_tables_wider_than_the_sequences(lengths, counts, heads, kv, extra, dtype, cache):
    """Work is cut by the table's width, so a wide one gives parts of few rows and of none: the same rows count."""
    r = Rows(lengths, counts, heads, kv, 128, 64, dtype, cache, True, extra)
    for window in (0, 200):
        r.run(r.prompt, window)
