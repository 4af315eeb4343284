"""Memory that an attention operator's results would share with what it reads: refused before any device is touched, and only where it is shared."""
import itertools
import random

import pytest
import torch

from paper_1202_3173_b200 import StrassenError, binding
from .test_attention_host import append, cache, decode, prompt

ALIAS, CUDA_ERROR = -4, -6
EIGHT = dict(type=binding.STRASSEN_E4M3, k_scale=3 << 20, v_scale=4 << 20)


def answer(call, c, **change):
    """The status of a call; None: it went through, or as far as the device, which this machine may not have."""
    try:
        call(c, **change)
    except StrassenError as e:
        return None if e.status == CUDA_ERROR else e.status
    return None


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no memory: without a device no kernel is launched")
@pytest.mark.parametrize("call,change", [
    # out over k and v, as parts of one wider tensor of 4 + 2 x 2 heads of 64, as neighbours and as one another's rows
    (append, dict(tokens=3, batch=3, q_row=512, k=16384 + 512, k_row=512, v=16384 + 768, v_row=512, out=16384 + 512, out_row=512)),
    (append, dict(tokens=3, batch=3, q_row=512, k=16384 + 512, k_row=512, v=16384 + 768, v_row=512, out=16384 + 768, out_row=512)),
    (append, dict(tokens=3, batch=3, q_row=512, k=16384 + 512, k_row=512, v=16384 + 768, v_row=512, out=16384 + 896, out_row=512)),
    (append, dict(out=32768)), (append, dict(out=32768 + 64)), (append, dict(out=65536 - 384)), (append, dict(out=65536 + 254)),
    # q moved by a head, by one element, by a row
    (append, dict(out=16384 + 128)), (append, dict(out=16384 + 2)), (append, dict(out=16384 - 510)), (append, dict(tokens=3, batch=3, out=16384 + 512)),
    # other distances between rows
    (append, dict(tokens=3, batch=3, out=32768 - 512, out_row=320)),
    # the table, the lengths, the frequencies
    (append, dict(out=4096)), (append, dict(out=4096 - 510)), (append, dict(out=8192)), (append, dict(out=12288 + 126)),
    (decode, dict(out=4096)), (decode, dict(out=8192 - 510)), (prompt, dict(out=12288 + 4)), (prompt, dict(out=8192)), (prompt, dict(out=4096 + 6))])
def test_results_over_what_is_read(call, change):
    change = {"table": 4096, "ld_table": 2, **change}
    assert answer(call, cache(), **change) == ALIAS, change


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no memory: without a device no kernel is launched")
@pytest.mark.parametrize("call", [append, decode, prompt])
@pytest.mark.parametrize("out", [3 << 20, (3 << 20) + 4 * 4 * 2 * 16 - 2, 4 << 20])
def test_results_over_the_scales(call, out):
    assert answer(call, cache(**EIGHT), out=out) == ALIAS
    assert answer(call, cache(**EIGHT), out=out + 4 * 4 * 2 * 16) is None


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no memory: without a device no kernel is launched")
def test_a_cache_over_what_is_read_or_over_itself():
    for change in (dict(table=(1 << 20) + 64), dict(lengths=2 << 20), dict(frequencies=(1 << 20) + 8188), dict(table=(3 << 20) + 8), dict(frequencies=4 << 20), dict(q=3 << 20), dict(v=4 << 20)):
        assert answer(append, cache(**EIGHT), **change) == ALIAS, change
    assert answer(append, cache(v=1 << 20)) == ALIAS
    assert answer(append, cache(**{**EIGHT, "v_scale": (3 << 20) + 8})) == ALIAS
    # keys and values side by side in one tensor
    assert answer(append, cache(v=(1 << 20) + 2048, page_stride=4096)) is None
    # where nothing is stored, keys may be the values
    assert answer(decode, cache(v=1 << 20)) is None and answer(prompt, cache(v=1 << 20)) is None


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no memory: without a device no kernel is launched")
def test_views_of_one_tensor_are_looked_at_element_by_element():
    """Random views of one wider tensor: refused if, and only if, an element of out is one of k, of v, or of q without being q."""
    rng = random.Random(5)
    seen = {True: 0, False: 0}
    for _ in range(4000):
        d, tokens = 8 * rng.randint(1, 3), rng.choice([1, 2, 3, 5])
        heads, kv = rng.randint(1, 4), rng.randint(1, 3)
        c = cache(kv_heads=kv, head_size=d, row_stride=d, head_stride=16 * d, page_stride=16 * kv * d)
        row, unit = rng.choice([d * rng.randint(1, 14), d * rng.randint(1, 14) + rng.randint(0, 9)]), rng.choice([d, d, 3 * d, d + rng.randint(0, 5)])
        views = []
        for n in (heads, kv, kv, heads):
            views.append((rng.randint(0, 16) * d + rng.choice([0, 0, rng.randint(0, 7)]), row, rng.choice([unit, unit, d, tokens * row]), n))
        if rng.random() < 0.3:
            views[3] = views[0]
        sets = [{at + t * r + h * s + i for t, h, i in itertools.product(range(tokens), range(n), range(d))} for at, r, s, n in views]
        want = bool(sets[3] & (sets[1] | sets[2])) or (bool(sets[3] & sets[0]) and views[3] != views[0])
        args = {}
        for name, (at, r, s, n) in zip(("q", "k", "v", "out"), views):
            args.update({name: (1 << 30) + 2 * at, name + "_row": r, name + "_head": s})
        # strides of dimensions of size 1 are nobody's: the views are the same then
        if views[3][0] == views[0][0] and sets[3] == sets[0] and (tokens == 1 or views[3][1] == views[0][1]) and (heads == 1 or views[3][2] == views[0][2]):
            want = bool(sets[3] & (sets[1] | sets[2]))
        got = answer(append, c, batch=tokens, tokens=tokens, heads=heads, rotary=0, frequencies=0, **args)
        assert got == (ALIAS if want else None), (views, tokens, d)
        seen[want] += 1
    assert min(seen.values()) > 500


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are no memory: without a device no kernel is launched")
def test_what_is_empty_shares_nothing():
    """A table without columns, wherever it points to; a cache without pages."""
    assert answer(decode, cache(), width=0, table=131072 + 64) is None
    assert answer(append, cache(), width=0, table=131072 + 64) is None
    assert answer(append, cache(), width=0, table=(1 << 20) + 64) is None
    assert answer(decode, cache(pages=0, type=binding.STRASSEN_E4M3, k_scale=131072 + 4, v_scale=131072 + 4)) is None
