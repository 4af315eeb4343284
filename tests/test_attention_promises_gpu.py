"""What the attention operators' documentation promises beyond their formulas: the codes of 8-bit rows, every row counted once, what is refused."""
import math
import os
import subprocess
import sys

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


@pytest.mark.parametrize("which", ["decode", "prompt"])
def test_a_workspace_over_what_is_read_is_refused(which):
    """Before anything is launched: over the table, the lengths and the cache's scales."""
    kv, d, page, width = 2, 64, 64, 4000
    cache = sw.PagedCache.empty(16, kv, d, page, E4M3)
    lengths, offsets = ints([100], [0, 4])
    q = torch.zeros(4 if which == "prompt" else 1, 4, d, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 9.0)
    table = torch.zeros(1, width, dtype=torch.int32, device="cuda")
    at = cache._at
    if which == "decode":
        need = binding.strassen_decode_attention_workspace_bytes(at, 1, 4, width)
    else:
        need = binding.strassen_prompt_attention_workspace_bytes(at, 1, 4, width, 4, 0)
    assert need > 0
    for over, inside in ((table, 0), (lengths, 0), (cache.k_scale, 0), (cache.v_scale, 0)) + (((offsets, 0),) if which == "prompt" else ()):
        ws = (over.data_ptr() + inside) // 256 * 256
        assert ws + need > over.data_ptr()
        with pytest.raises(StrassenError) as e:
            if which == "decode":
                binding.strassen_decode_attention(at, 1, table.data_ptr(), width, width, lengths.data_ptr(), 0, 4, q.data_ptr(), 4 * d, d, out.data_ptr(), 4 * d, d, 0.125, 0, ws, need)
            else:
                binding.strassen_prompt_attention(at, 1, table.data_ptr(), width, width, lengths.data_ptr(), offsets.data_ptr(), 4, 0, 4, q.data_ptr(), 4 * d, d, out.data_ptr(), 4 * d, d,
                                                  0.125, 0, ws, need)
        assert e.value.status == -4 and "workspace" in str(e.value)
    torch.cuda.synchronize()
    assert bool((out == 9).all())


def test_results_over_keys_or_values_of_one_product_are_refused():
    """Queries, keys and values as views of one product's rows: turned in place, but not over the keys or values beside them."""
    rows = torch.randn(20, 4 + 2 + 2, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    q, k, v = rows[:, :4], rows[:, 4:6], rows[:, 6:]
    cache = sw.PagedCache.empty(2, 2, 64, 16)
    table, lengths, offsets = ints([[0, 1]], [20], [0, 20])
    keep = rows.clone()
    for out in (rows[:, 2:6], rows[:, 4:], rows[:, 1:5]):
        with pytest.raises(StrassenError):
            sw.rotate_append(q, k, v, cache, table, lengths, None, offsets, out=out)
    torch.cuda.synchronize()
    assert torch.equal(rows, keep)
    assert sw.rotate_append(q, k, v, cache, table, lengths, None, offsets, out=q) is q and torch.equal(rows, keep)
    # every head's query, key and value side by side
    each = keep[:, :6].reshape(20, 2, 3, 64).clone()
    want = sw.rotate_append(each[:, :, 0].contiguous(), each[:, :, 1], each[:, :, 2], cache, table, lengths, None, offsets)
    assert torch.equal(sw.rotate_append(each[:, :, 0], each[:, :, 1], each[:, :, 2], cache, table, lengths, None, offsets, out=each[:, :, 0]), want)
    with pytest.raises(StrassenError):
        sw.rotate_append(each[:, :, 0], each[:, :, 1], each[:, :, 2], cache, table, lengths, None, offsets, out=each[:, :, 2])


@pytest.mark.parametrize("cache_type", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("kv,pages,page", [(1, 70, 16), (1, 1, 1024), (2, 1, 1024), (1, 9, 128), (3, 70, 16)])
def test_one_key_head_or_one_page_wherever_pages_lie(kv, pages, page, cache_type):
    """Rows one after another and pages with room between them are brought by different copies: the same bits.  (A stride of a dimension of one says nothing.)"""
    d, n = 64, 1000
    g = torch.Generator("cuda").manual_seed(pages)
    table = torch.full((1, max(pages, -(-n // page)) + 1), -1, dtype=torch.int32, device="cuda")
    used = -(-n // page)
    table[0, :used] = torch.randperm(pages, device="cuda", generator=g)[:used]
    table[0, used // 2] = pages if pages > 1 else table[0, used // 2]                # a page that is not there
    lengths, offsets = ints([n], [0, 300])
    q = torch.randn(300, 4 * kv, d, device="cuda", generator=g).bfloat16()
    k, v = (torch.randn(pages, kv, page, d, device="cuda", generator=g).to(cache_type) for _ in range(2))
    scales = [torch.rand(pages, kv, page, device="cuda", generator=g) + 0.5 if cache_type == E4M3 else None for _ in range(2)]

    def wide(x, shape, strides, total):
        t = torch.full((total,), math.nan, device="cuda").to(cache_type)
        t = torch.as_strided(t, shape, strides)
        (t.view(torch.uint8) if cache_type == E4M3 else t).copy_(x.view(torch.uint8) if cache_type == E4M3 else x)
        return t

    got = []
    shape = (pages, kv, page, d)
    for strides in ((kv * page * d, page * d, d, 1), (kv * page * d + 64, page * d, d, 1), (kv * page * (d + 32), page * (d + 32), d + 32, 1), (7 * kv * page * d, 7 * page * d, d, 1)):
        total = sum((n - 1) * s for n, s in zip(shape, strides)) + 1
        cache = sw.PagedCache(wide(k, shape, strides, total), wide(v, shape, strides, total), *scales)
        got.append((sw.prompt_attention(q, cache, table, lengths, offsets), sw.prompt_attention(q, cache, table, lengths, offsets, window=77), sw.decode_attention(q[-1:], cache, table, lengths)))
    assert bool(torch.isfinite(got[0][0]).all())
    for other in got[1:]:
        for a, b in zip(got[0], other):
            assert torch.equal(a, b)


@pytest.mark.parametrize("cache_type", [torch.bfloat16, E4M3])
def test_tiles_without_rows_wait_for_the_whole_block(cache_type):
    """300 sequences of one token behind 120000 rows (the same pages): every block of two tiles of queries has one without rows, which waits for all of the other's."""
    d, page, n, batch = 64, 1024, 120000, 300
    pages = -(-n // page)
    k = torch.zeros(pages, 1, page, d, device="cuda").to(cache_type)
    v = torch.zeros(pages, 1, page, d, device="cuda")
    v[:, :, ::2, 0] = 1.0                                    # every second row: its mean is 1/2
    v[0, 0, 0, 1] = 256.0                                    # the first and the last row
    v[-1, 0, (n - 1) % page, 2] = 256.0
    scales = [torch.ones(pages, 1, page, device="cuda") if cache_type == E4M3 else None for _ in range(2)]
    cache = sw.PagedCache(k, v.to(cache_type), *scales)
    table = torch.arange(pages, device="cuda", dtype=torch.int32)[None].expand(batch, -1).contiguous()
    lengths = torch.full((batch,), n, dtype=torch.int32, device="cuda")
    offsets = torch.arange(batch + 1, device="cuda", dtype=torch.int32)
    q = torch.randn(batch, 2, d, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).bfloat16()
    assert binding.strassen_prompt_attention_workspace_bytes(cache._at, batch, 2, pages, batch, 0) == 0
    out = sw.prompt_attention(q, cache, table, lengths, offsets)
    binding.strassen_device_status()
    want = torch.zeros(d, dtype=torch.float64, device="cuda")
    want[0], want[1], want[2] = 0.5, 256 / n, 256 / n
    # equal weights, exact in 16 bits; sums in 32 bits of 2^17 terms and one rounding to bf16
    assert bool(((out.double() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -18)).all())


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("cache_type", [torch.bfloat16, torch.float16, E4M3])
@pytest.mark.parametrize("window", [0, 2000])
def test_infinite_values_behind_many_rows_in_parts(bad, cache_type, window):
    """The last row's value is infinite, and its score so far above all others that these weigh 0 in 32 bits; with a window so is the value of a row that the first two tokens see
    alone, in another part of the cut.  A token that sees such a value has it, as the formula has, whatever its parts weigh; one that does not is as ever."""
    d, page, n, count = 64, 64, 20000, 4
    pages = -(-n // page)
    k, v = (torch.zeros(pages, 1, page, d, device="cuda") for _ in range(2))
    rows = [n - 1] + ([n - count - window + 2] if window else [])
    k[(n - 1) // page, 0, (n - 1) % page, 0] = 256.0
    v[..., 1] = 1.0
    scales = [torch.ones(pages, 1, page, device="cuda") if cache_type == E4M3 else None for _ in range(2)]
    v = v.to(cache_type)
    for r in rows:
        if cache_type == E4M3:
            scales[1][r // page, 0, r % page] = bad           # column 1 infinite; 0 times that, in the others, is NaN
        else:
            v[r // page, 0, r % page, 1] = bad
    cache = sw.PagedCache(k.to(cache_type), v, *scales)
    q = torch.zeros(count, 2, d, dtype=torch.float16 if cache_type == torch.float16 else torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    table = torch.arange(pages, device="cuda", dtype=torch.int32)[None]
    lengths, offsets = ints([n], [0, count])
    assert binding.strassen_prompt_attention_workspace_bytes(cache._at, 1, 2, pages, count, window) > 0
    out = sw.prompt_attention(q, cache, table, lengths, offsets, scale=1.0, window=window).double()
    for i in range(count):
        p = n - count + i
        sees = [r for r in rows if r <= p and (not window or r > p - window)]
        assert len(sees) == ((i == 3) if not window else (1, 1, 0, 1)[i])
        if sees:
            assert torch.equal(out[i, :, 1].nan_to_num(1.5, 2.5, -2.5), torch.full((2,), bad, dtype=torch.float64, device="cuda").nan_to_num(1.5, 2.5, -2.5)), i
        else:
            assert bool(((out[i, :, 1] - 1.0).abs() <= 2.0 ** -8 + 2.0 ** -18).all())
        if cache_type != E4M3 or not sees:
            assert not bool(out[i, :, 0].any()) and not bool(out[i, :, 2:].any())


FIRST = """
import torch, paper_1202_3173_b200 as sw
cache = sw.PagedCache.empty(16, 8, 128, 64)
cache.k.normal_(), cache.v.normal_()
q = torch.randn(1, 32, 128, device="cuda").bfloat16()
table = torch.arange(16, dtype=torch.int32, device="cuda")[None]
lengths = torch.tensor([1000], dtype=torch.int32, device="cuda")
out, graph, stream = torch.zeros_like(q), torch.cuda.CUDAGraph(), torch.cuda.Stream()
torch.cuda.synchronize()
with torch.cuda.graph(graph, stream=stream):
    sw.decode_attention(q, cache, table, lengths, out=out)
graph.replay()
torch.cuda.synchronize()
want = sw.decode_attention(q, cache, table, lengths)
assert torch.equal(out, want) and bool(out.any())
print("ok")
"""


def test_the_first_call_of_a_process_may_be_captured():
    """What a call asks the device once (the largest cluster, the shared memory) it may ask while a graph is being captured."""
    done = subprocess.run([sys.executable, "-c", FIRST], capture_output=True, text=True, timeout=120, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert done.returncode == 0 and done.stdout.strip() == "ok", done.stderr[-2000:]
