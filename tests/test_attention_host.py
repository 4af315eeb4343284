"""Host side of the attention operators: refusals that need no device."""
import ctypes

import pytest

from paper_1202_3173_b200 import StrassenError, binding

GOOD = dict(type=binding.STRASSEN_BF16, kv_heads=2, head_size=64, page_size=16, pages=4, k=1 << 20, v=2 << 20, page_stride=2048, head_stride=1024, row_stride=64,
            k_scale=0, v_scale=0)


def cache(**change):
    return binding.strassen_paged_cache(**{**GOOD, **change})


def append(c, **change):
    a = dict(batch=1, table=4096, ld_table=2, width=2, lengths=8192, offsets=0, tokens=1, type=0, heads=4, q=16384, q_row=256, q_head=64, k=32768, k_row=128, k_head=64, v=65536,
             v_row=128, v_head=64, out=131072, out_row=256, out_head=64, frequencies=12288, rotary=64, interleaved=False)
    a.update(change)
    binding.strassen_rotate_append(ctypes.addressof(c), **a)


def decode(c, **change):
    a = dict(batch=1, table=4096, ld_table=2, width=2, lengths=8192, type=0, heads=4, q=16384, q_row=256, q_head=64, out=131072, out_row=256, out_head=64, scale=0.125, window=0)
    a.update(change)
    binding.strassen_decode_attention(ctypes.addressof(c), **a)


def prompt(c, **change):
    a = dict(batch=1, table=4096, ld_table=2, width=2, lengths=8192, offsets=12288, tokens=3, type=0, heads=4, q=16384, q_row=256, q_head=64, out=131072, out_row=256, out_head=64,
             scale=0.125, window=0)
    a.update(change)
    binding.strassen_prompt_attention(ctypes.addressof(c), **a)


@pytest.mark.parametrize("status,change", [
    (-1, dict(type=2)), (-1, dict(type=7)), (-1, dict(kv_heads=0)), (-1, dict(kv_heads=1025)), (-1, dict(head_size=0)), (-1, dict(head_size=4)), (-1, dict(head_size=68)),
    (-1, dict(head_size=136)), (-1, dict(page_size=0)), (-1, dict(page_size=4)), (-1, dict(page_size=24)), (-1, dict(page_size=2048)), (-1, dict(pages=-1)), (-1, dict(pages=2 ** 31)),
    (-1, dict(k=0)), (-1, dict(v=0)), (-1, dict(page_stride=32)), (-1, dict(head_stride=56)), (-1, dict(row_stride=0)), (-5, dict(row_stride=65)), (-5, dict(page_stride=2052)),
    (-5, dict(k=(1 << 20) + 8)), (-5, dict(v=(2 << 20) + 2)), (-1, dict(k_scale=4096)), (-1, dict(type=3)), (-1, dict(type=3, k_scale=4096)), (-5, dict(type=3, k_scale=4097, v_scale=4096)),
    (-1, dict(type=3, k_scale=4096, v_scale=4096, head_size=72, row_stride=80))])
@pytest.mark.parametrize("call", [append, decode, prompt])
def test_caches_are_checked_before_any_device_is_touched(call, status, change):
    with pytest.raises(StrassenError) as e:
        call(cache(**change))
    assert e.value.status == status and str(e.value), change


@pytest.mark.parametrize("call,status,change", [
    (append, -1, dict(batch=-1)), (append, -1, dict(tokens=2)), (append, -1, dict(lengths=0)), (append, -1, dict(table=0)), (append, -1, dict(batch=2, tokens=2, ld_table=1)),
    (append, -1, dict(type=2)), (append, -1, dict(type=1)), (append, -1, dict(heads=-1)), (append, -1, dict(heads=1025)), (append, -1, dict(rotary=63)), (append, -1, dict(rotary=66)),
    (append, -1, dict(rotary=0)), (append, -1, dict(frequencies=0)), (append, -1, dict(q=0)), (append, -1, dict(k=0)), (append, -1, dict(v=0)), (append, -1, dict(out=0)),
    (append, -1, dict(heads=0)), (append, -1, dict(k_head=32)), (append, -1, dict(q_head=63)), (append, -5, dict(k=32769)), (append, -5, dict(lengths=8194)), (append, -5, dict(frequencies=12290)),
    (append, -4, dict(q=1 << 20)), (append, -4, dict(out=2 << 20)), (append, -4, dict(out=16384, out_head=128)),
    (decode, -1, dict(heads=3)), (decode, -1, dict(heads=0)), (decode, -1, dict(scale=float("nan"))), (decode, -1, dict(scale=float("inf"))), (decode, -1, dict(window=-1)),
    (decode, -1, dict(q=0)), (decode, -1, dict(out=0)), (decode, -1, dict(width=-1)), (decode, -1, dict(type=3)), (decode, -5, dict(q=16385)), (decode, -5, dict(table=4098)),
    (decode, -4, dict(out=16384)), (decode, -4, dict(out=1 << 20)),
    (prompt, -1, dict(offsets=0)), (prompt, -1, dict(q_row=32)), (prompt, -1, dict(tokens=-1)), (prompt, -5, dict(offsets=12289)), (prompt, -4, dict(out=16384 + 512))])
def test_arguments_are_checked_before_any_device_is_touched(call, status, change):
    with pytest.raises(StrassenError) as e:
        call(cache(), **change)
    assert e.value.status == status and str(e.value), change


def test_no_cache_and_nothing_to_do():
    with pytest.raises(StrassenError):
        binding.strassen_decode_attention(0, 1, 4096, 2, 2, 8192, 0, 4, 16384, 256, 64, 131072, 256, 64, 0.1, 0)
    append(cache(), batch=0, tokens=0)
    decode(cache(), batch=0)
    prompt(cache(), batch=0, tokens=0)
    prompt(cache(), tokens=0, q=0, out=0)
    assert binding.strassen_decode_attention_workspace_bytes(0, 1, 4, 2) == 0
    assert binding.strassen_prompt_attention_workspace_bytes(0, 1, 4, 2, 1, 0) == 0


def test_the_package_offers_the_operators():
    import paper_1202_3173_b200 as sw
    for name in ("PagedCache", "SelfAttention", "rotate_append", "decode_attention", "prompt_attention"):
        assert name in sw.__all__ and callable(getattr(sw, name))
