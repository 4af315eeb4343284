"""Attention of a served model on torch tensors, over a paged cache of keys and values.

The work is done by the kernels behind ``strassen_rotate_append``, ``strassen_decode_attention`` and ``strassen_prompt_attention``
(``include/strassen_b200.h`` has their formulas and what they do with lengths, pages and offsets of every kind); here are the checks of shapes, types and
devices, the memory and the current stream.  ``SelfAttention`` runs them together as one block, beside ``FeedForward``;
``python -m paper_1202_3173_b200.attention`` tries it out.

Row j of sequence b lies in page ``table[b, j // page_size]``, slot ``j % page_size``.  ``lengths[b]`` counts the sequence's rows with its new ones, which are the
last ``offsets[b + 1] - offsets[b]``: rows ``offsets[b]`` to ``offsets[b + 1] - 1`` of q.  Without offsets each sequence has one new token.  ``table``,
``lengths`` and ``offsets`` are int32 CUDA tensors that the kernels read, so that a captured graph can be replayed for other lengths; which pages are
handed to which sequence is the caller's to decide.  How work is cut goes by the table's width, which the host sees: a table no wider than the longest sequence needs is the
fastest (prompts in one for many times their rows take several times as long and up to some 300 MB of workspace).  Rows that belong to no sequence are not written (what a new result holds for them is not defined).

Calls are enqueued on the current stream and can be captured into a CUDA graph.  The operators serve a model and have no backward pass: tensors that require
grad are refused unless gradients are off (``torch.no_grad()``), tensors with forward-mode tangents always.  Tensors that are written count as modified in place.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import binding
from .feed_forward import _OUT_TYPES, _TYPES, E4M3, W4Matrix, _call, _current_device, _forward_mode, _gradients_off, _packed, _tangents_off, _written, quantize_w4, rms_norm_quant

__all__ = ["PagedCache", "SelfAttention", "rotate_append", "decode_attention", "prompt_attention"]

_INT = torch.int32
_HERE = contextlib.nullcontext()


class PagedCache:
    """Keys and values in pages: ``k`` and ``v`` (pages, kv_heads, page_size, head_size), bfloat16, float16 or float8_e4m3fn; for 8 bits also ``k_scale``
    and ``v_scale`` (float32, pages, kv_heads, page_size), so that a row is k * k_scale.

    ``page_size`` is a power of two, 8 .. 1024; ``head_size`` a multiple of 8 (8 bits: 16) up to 128.  k and v may be views with other orders of pages, heads and
    rows, as long as rows are contiguous, strides and addresses are multiples of 16 bytes, and both have the same strides."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if _forward_mode():
            _tangents_off(k=k, v=v, k_scale=k_scale, v_scale=v_scale)
        if k.dim() != 4 or k.dtype not in _CACHE_TYPES or not k.is_cuda:
            raise ValueError("k must be a CUDA tensor (pages, kv_heads, page_size, head_size) of one of %s, not %s %s on %s"
                             % (", ".join(str(t) for t in _CACHE_TYPES), k.dtype, tuple(k.shape), k.device))
        if v.shape != k.shape or v.dtype != k.dtype or v.device != k.device or v.stride() != k.stride():
            raise ValueError("v must be as k: %s %s on %s with strides %s, not %s %s on %s with %s"
                             % (k.dtype, tuple(k.shape), k.device, k.stride(), v.dtype, tuple(v.shape), v.device, v.stride()))
        if (k_scale is None) != (k.dtype != E4M3) or (v_scale is None) != (k.dtype != E4M3):
            raise ValueError("k_scale and v_scale go with a cache in 8 bits, and only with one")
        self.pages, self.kv_heads, self.page_size, self.head_size = k.shape
        if k.numel() and k.stride(3) != 1:
            raise ValueError("the rows of k and v must be contiguous (last stride 1)")
        if self.page_size & (self.page_size - 1) or not 8 <= self.page_size <= 1024:
            raise ValueError("page_size must be a power of two, 8 .. 1024, not %d" % self.page_size)
        unit = 16 // k.element_size()
        if self.head_size % unit or not 1 <= self.head_size <= 128:
            raise ValueError("head_size must be a multiple of %d up to 128, not %d" % (unit, self.head_size))
        if not 1 <= self.kv_heads <= 1024:
            raise ValueError("kv_heads must be 1 .. 1024, not %d" % self.kv_heads)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.dtype, self.device, self._index = k.dtype, k.device, k.get_device()
        for name, t in (("k", k), ("v", v)):
            if t.requires_grad:
                _gradients_off(name)
            if t.data_ptr() % 16 or any(s % unit for s, n in zip(t.stride()[:3], t.shape[:3]) if n > 1):
                raise ValueError("%s must start at a multiple of 16 bytes, and so must each of its rows" % name)
            if any(s < self.head_size for s, n in zip(t.stride()[:3], t.shape[:3]) if n > 1):
                raise ValueError("the rows of %s overlap" % name)
        ks, vs = (_packed(n, t, k.shape[:3], torch.float32, self._index) if t is not None else 0 for n, t in (("k_scale", k_scale), ("v_scale", v_scale)))
        self._kind = _CACHE_TYPES[k.dtype]
        row = k.stride(2) if self.page_size > 1 else self.head_size
        self._c = binding.strassen_paged_cache(self._kind, self.kv_heads, self.head_size, self.page_size, self.pages, k.data_ptr(), v.data_ptr(),
                                               k.stride(0), k.stride(1), row, ks, vs)
        self._at = ctypes.addressof(self._c)
        self._decode_workspace = {}      # by heads, sequences and the table's width

    @classmethod
    def empty(cls, pages, kv_heads, head_size, page_size=64, dtype=torch.bfloat16, device="cuda"):
        """A cache in new memory, one page after another."""
        shape = (int(pages), int(kv_heads), int(page_size), int(head_size))
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        scales = [torch.empty(shape[:3], dtype=torch.float32, device=device) if dtype == E4M3 else None for _ in range(2)]
        return cls(k, v, *scales)

    @property
    def nbytes(self):
        """Device memory of the cache's values and scales."""
        return sum(t.numel() * t.element_size() for t in (self.k, self.v, self.k_scale, self.v_scale) if t is not None)


_CACHE_TYPES = {torch.bfloat16: _TYPES[torch.bfloat16], torch.float16: _TYPES[torch.float16], E4M3: _TYPES[E4M3]}


def _heads(name, t, shape, dtype, index):
    """Strides of the rows and heads of ``t`` after checking it."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        raise ValueError("%s must be a %s tensor of shape %s on cuda:%d, not %s %s on %s" % (name, dtype, tuple(shape), index, t.dtype, tuple(t.shape), t.device))
    if t.requires_grad:
        _gradients_off(name)
    row, head, step = t.stride()
    if step != 1 and shape[2] != 1:
        raise ValueError("the heads of %s must be contiguous (last stride 1)" % name)
    return row, head


def _sequences(q, cache, table, lengths, offsets):
    """(batch, table's address, its leading dimension, width, lengths' address, offsets' address) after checking them."""
    index = cache._index
    if lengths.dtype is not _INT or lengths.get_device() != index or lengths.dim() != 1 or not lengths.is_contiguous():
        raise ValueError("lengths must be a contiguous int32 tensor of one dimension on cuda:%d, not %s %s on %s" % (index, lengths.dtype, tuple(lengths.shape), lengths.device))
    batch = lengths.shape[0]
    if table.dtype is not _INT or table.get_device() != index or table.dim() != 2 or table.shape[0] != batch:
        raise ValueError("table must be an int32 tensor of %d rows on cuda:%d, not %s %s on %s" % (batch, index, table.dtype, tuple(table.shape), table.device))
    ld, step = table.stride()
    width = table.shape[1]
    if step != 1 and width > 1:
        raise ValueError("the rows of table must be contiguous (last stride 1)")
    if offsets is None:
        if q.shape[0] != batch:
            raise ValueError("%d rows for %d sequences of one new token: offsets say where each one's are" % (q.shape[0], batch))
        return batch, table.data_ptr(), ld, width, lengths.data_ptr(), 0
    if offsets.dtype is not _INT or offsets.get_device() != index or offsets.shape != (batch + 1,) or not offsets.is_contiguous():
        raise ValueError("offsets must be a contiguous int32 tensor of %d entries on cuda:%d, not %s %s on %s" % (batch + 1, index, offsets.dtype, tuple(offsets.shape), offsets.device))
    return batch, table.data_ptr(), ld, width, lengths.data_ptr(), offsets.data_ptr()


def _type_of(q, cache, name="q"):
    kind = _OUT_TYPES.get(q.dtype)
    if kind is None or q.dim() != 3:
        raise ValueError("%s must be a CUDA tensor (tokens, heads, head_size) in bfloat16 or float16, not %s %s" % (name, q.dtype, tuple(q.shape)))
    if cache.dtype is not E4M3 and cache.dtype is not q.dtype:
        raise ValueError("%s is %s, the cache %s" % (name, q.dtype, cache.dtype))
    return kind


def rotate_append(q, k, v, cache, table, lengths, frequencies=None, offsets=None, interleaved=False, out=None):
    """Rotary embedding of the new tokens' queries and keys, and their keys and values stored into ``cache``: the turned queries.

    ``q``: (tokens, heads, head_size) or None; ``k``, ``v``: (tokens, kv_heads, head_size); any of them may be views of one wider tensor.  ``frequencies``: float32,
    one for each pair that turns (up to head_size / 2); pair f of a token at position p turns by p * frequencies[f].  Pairs are the values f and f + n of the first
    2 n of a row, or, ``interleaved``, 2 f and 2 f + 1.  Without frequencies nothing turns.  ``out``: to write the turned queries to; may be ``q`` itself."""
    if _forward_mode():
        _tangents_off(q=q, k=k, v=v, frequencies=frequencies, out=out)
    kind = _type_of(k, cache, "k")
    index, tokens, size = cache._index, k.shape[0], cache.head_size
    seq = _sequences(k, cache, table, lengths, offsets)
    shape = (tokens, cache.kv_heads, size)
    k_row, k_head = _heads("k", k, shape, k.dtype, index)
    v_row, v_head = _heads("v", v, shape, k.dtype, index)
    heads = qp = q_row = q_head = op = o_row = o_head = 0
    given = out
    if q is not None:
        if q.dim() != 3:
            raise ValueError("q must be (tokens, heads, head_size), not %s" % (tuple(q.shape),))
        heads = q.shape[1]
        q_row, q_head = _heads("q", q, (tokens, heads, size), k.dtype, index)
        if out is None:
            out = torch.empty(tokens, heads, size, dtype=k.dtype, device=cache.device)
        o_row, o_head = _heads("out", out, (tokens, heads, size), k.dtype, index)
        qp, op = q.data_ptr(), out.data_ptr()
    elif out is not None:
        raise ValueError("out is for the turned queries, and there is no q")
    rotary = fp = 0
    if frequencies is not None:
        if frequencies.dim() != 1 or not 1 <= frequencies.shape[0] <= size // 2:
            raise ValueError("frequencies must be 1 .. %d numbers, not %s" % (size // 2, tuple(frequencies.shape)))
        rotary, fp = 2 * frequencies.shape[0], _packed("frequencies", frequencies, frequencies.shape, torch.float32, index)
    batch, table_at, ld, width, lengths_at, offsets_at = seq
    _call(index, binding.strassen_rotate_append, cache._at, batch, table_at, ld, width, lengths_at, offsets_at, tokens, kind, heads, qp, q_row, q_head,
          k.data_ptr(), k_row, k_head, v.data_ptr(), v_row, v_head, op, o_row, o_head, fp, rotary, interleaved)
    _written((cache.k, cache.v) + ((cache.k_scale, cache.v_scale) if cache.k_scale is not None else ()) + (() if given is None else (given,)))
    return out


def _attention(q, cache, table, lengths, offsets, scale, window, out):
    if _forward_mode():
        _tangents_off(q=q, out=out)
    kind = _type_of(q, cache)
    index = cache._index
    batch, table_at, ld, width, lengths_at, offsets_at = _sequences(q, cache, table, lengths, offsets)
    shape = q.shape
    tokens, heads, size = shape
    q_row, q_head = _heads("q", q, (tokens, heads, cache.head_size), q.dtype, index)
    given = out
    if out is None:
        out = torch.empty(shape, dtype=q.dtype, device=cache.device)
    o_row, o_head = _heads("out", out, shape, q.dtype, index)
    if scale is None:
        scale = size ** -0.5
    ws = need = 0
    if offsets is not None and (q.data_ptr() | 2 * q_row | 2 * q_head) % 16:
        q = torch.empty(shape, dtype=q.dtype, device=cache.device).copy_(q)         # prompts are read in boxes that start at multiples of 16 bytes
        q_row, q_head, _ = q.stride()
    if offsets is None:
        sizes = heads, batch, width
        need = cache._decode_workspace.get(sizes)
        if need is None:                                        # the size goes by these alone
            if len(cache._decode_workspace) >= 4096:
                cache._decode_workspace.clear()
            with torch.cuda.device(index):
                need = binding.strassen_decode_attention_workspace_bytes(cache._at, batch, heads, width)
            cache._decode_workspace[sizes] = need
    else:
        with torch.cuda.device(index) if index != _current_device() else _HERE:
            need = binding.strassen_prompt_attention_workspace_bytes(cache._at, batch, heads, width, tokens, window)
    if need:
        # from the allocator of the current stream, which the call is enqueued on: free again when the call is done
        workspace = torch.empty(need, dtype=torch.uint8, device=cache.device)
        ws = workspace.data_ptr()
    if offsets is None:
        _call(index, binding.strassen_decode_attention, cache._at, batch, table_at, ld, width, lengths_at, kind, heads, q.data_ptr(), q_row, q_head, out.data_ptr(),
              o_row, o_head, scale, window, ws, need)
    else:
        _call(index, binding.strassen_prompt_attention, cache._at, batch, table_at, ld, width, lengths_at, offsets_at, tokens, kind, heads, q.data_ptr(), q_row, q_head,
              out.data_ptr(), o_row, o_head, scale, window, ws, need)
    if given is not None:
        _written((given,))
    return out


def decode_attention(q, cache, table, lengths, scale=None, window=0, out=None):
    """Attention of one new token a sequence: row b of ``q`` (batch, heads, head_size) over the first ``lengths[b]`` rows of sequence b, with a ``window`` over the
    last of them.  ``heads`` is a multiple of the cache's kv_heads; neighbouring heads share a key head.  ``scale``: of the scores, 1 / sqrt(head_size)."""
    return _attention(q, cache, table, lengths, None, scale, window, out)


def prompt_attention(q, cache, table, lengths, offsets, scale=None, window=0, out=None):
    """Attention of the new tokens of each sequence (rows ``offsets[b]`` .. ``offsets[b + 1] - 1`` of ``q``), each over the rows up to its own position, with a
    ``window`` over the last of those.  Whole prompts, their next parts behind what the cache has already, or few tokens."""
    if offsets is None:
        raise ValueError("prompt_attention needs offsets; decode_attention is for one new token a sequence")
    return _attention(q, cache, table, lengths, offsets, scale, window, out)


class SelfAttention:
    """One served attention block:  h = x + residual;  y = o(attention(q, k, v)) with q, k, v = qkv(n) and n the norm of h.

    ``qkv`` is a W4Matrix of (heads + 2 kv_heads) * head_size rows (queries above keys above values) over the model's width, ``o`` one of the width's rows over
    heads * head_size.  ``frequencies``, ``interleaved``: as ``rotate_append``; ``window``, ``scale``: as the attention."""

    def __init__(self, norm_weight, qkv, o, heads, frequencies=None, eps=1e-6, interleaved=False, scale=None, window=0):
        if o.k % heads or qkv.n <= o.k or (qkv.n - o.k) % (2 * (o.k // heads)) or o.n != qkv.k or tuple(norm_weight.shape) != (qkv.k,):
            raise ValueError("a block of width %d and %d heads needs a norm of that size, qkv ((heads + 2 kv_heads) * head_size x %d) and o (%d x heads * head_size); got %s, %d x %d and %d x %d"
                             % (qkv.k, heads, qkv.k, qkv.k, tuple(norm_weight.shape), qkv.n, qkv.k, o.n, o.k))
        self.norm_weight, self.qkv, self.o, self.heads, self.eps = norm_weight, qkv, o, int(heads), eps
        self.head_size = o.k // self.heads
        self.kv_heads = (qkv.n - o.k) // (2 * self.head_size)
        self.frequencies, self.interleaved, self.scale, self.window = frequencies, interleaved, scale, window

    def __call__(self, x, residual, cache, table, lengths, offsets=None):
        """(y, h), both of x's type, for rows x of new tokens (one a sequence, or as offsets say): the block's output, to be added to the residual stream h by the
        next norm.  The new keys and values are in the cache afterwards.  Beside float32 rows the block works in the cache's type (bfloat16 for one in 8 bits)."""
        if (cache.kv_heads, cache.head_size) != (self.kv_heads, self.head_size):
            raise ValueError("the block has %d key heads of %d, the cache %d of %d" % (self.kv_heads, self.head_size, cache.kv_heads, cache.head_size))
        n, s, h = rms_norm_quant(x, self.norm_weight, self.eps, residual=residual)
        dtype = x.dtype if x.dtype is not torch.float32 else cache.dtype if cache.dtype is not E4M3 else torch.bfloat16
        rows = self.qkv(n, s, dtype=dtype).view(x.shape[0], self.heads + 2 * self.kv_heads, self.head_size)
        q, k, v = rows[:, :self.heads], rows[:, self.heads:self.heads + self.kv_heads], rows[:, self.heads + self.kv_heads:]
        rotate_append(q, k, v, cache, table, lengths, self.frequencies, offsets, self.interleaved, out=q)
        a = _attention(q, cache, table, lengths, offsets, self.scale, self.window, None)
        return self.o(a.view(x.shape[0], self.o.k)).to(x.dtype), h


def main():
    """A block of width 4096 with 32 heads over 8 key heads: a prompt, then one token at a time, against the same block in 32 bits."""
    width, heads, kv, d, group = 4096, 32, 8, 128, 128
    g = torch.Generator("cuda").manual_seed(0)
    weights, plain = [], []
    for n, k in (((heads + 2 * kv) * d, width), (width, heads * d)):
        q, s, z = quantize_w4(torch.randn(n, k, device="cuda", generator=g) * 0.02, group)
        weights.append(W4Matrix(q, s, z, k=k, group=group))
        nibbles = torch.stack([q & 15, q >> 4], -1).view(n, k).float()
        plain.append(s.float().repeat_interleave(group, 1) * (nibbles - z.float().repeat_interleave(group, 1)))
    frequencies = 500000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)
    block = SelfAttention(torch.ones(width, device="cuda", dtype=torch.bfloat16), *weights, heads, frequencies)
    prompt, steps = 700, 4
    cache = PagedCache.empty(16, kv, d, 64)
    table = torch.randperm(16, device="cuda", generator=g).to(torch.int32)[None]
    x, r = (torch.randn(prompt + steps, width, device="cuda", generator=g).bfloat16() for _ in range(2))
    got = []
    for i, end in enumerate([prompt] + [prompt + j + 1 for j in range(steps)]):
        first = 0 if i == 0 else end - 1
        lengths, offsets = torch.tensor([end], dtype=torch.int32, device="cuda"), torch.tensor([0, end - first], dtype=torch.int32, device="cuda")
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for repeat in range(4):
            if repeat == 1:
                start.record()
            y, _ = block(x[first:end], r[first:end], cache, table, lengths, offsets if i == 0 else None)
        stop.record()
        torch.cuda.synchronize()
        got.append(y)
        print("%4d new tokens of %d: %7.1f us a block" % (end - first, end, start.elapsed_time(stop) / 3 * 1e3))
    n = x.float() + r.float()
    n = n * (n.square().mean(-1, keepdim=True) + block.eps).rsqrt()
    rows = (n @ plain[0].t()).view(prompt + steps, -1, d)
    angle = torch.arange(prompt + steps, device="cuda")[:, None, None] * frequencies
    a, b = rows[:, :heads + kv].chunk(2, -1)
    turned = torch.cat([a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()], -1)
    q, k, v = turned[:, :heads], turned[:, heads:].repeat_interleave(heads // kv, 1), rows[:, heads + kv:].repeat_interleave(heads // kv, 1)
    score = torch.einsum("qhd,jhd->hqj", q, k) * d ** -0.5
    score = score + torch.full_like(score, float("-inf")).triu(1)
    want = torch.einsum("hqj,jhd->qhd", score.softmax(-1), v).flatten(1) @ plain[1].t()
    got = torch.cat(got).float()
    for name, part in (("prompt", slice(0, prompt)), ("single tokens", slice(prompt, None))):
        print("%s: %.3f of the 32-bit block's output is the rounding to 8 bits" % (name, float((got[part] - want[part]).norm() / want[part].norm())))


if __name__ == "__main__":
    main()
