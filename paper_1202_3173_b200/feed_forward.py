"""Feed-forward operators of a served model on torch tensors: rows of activations in 8 bits, weights in 4.

The work is done by the kernels behind ``strassen_rms_norm_quant``, ``strassen_silu_mul_quant`` and ``strassen_w4_matmul``
(``include/strassen_b200.h`` has their formulas); here are the checks of shapes, types and devices, the memory and the
current stream.  ``FeedForward`` runs them together as one block; ``python -m paper_1202_3173_b200.feed_forward`` tries it out.

Rows are 2-D CUDA tensors whose last dimension is contiguous; rows may be any distance apart (views of wider tensors).  Calls are
enqueued on the current stream, allocate nothing when ``out`` is given, and can be captured into a CUDA graph.

The operators serve a model and have no backward pass: tensors that require grad are refused unless gradients are off
(``torch.no_grad()``), tensors with forward-mode tangents always.  Tensors that are written count as modified in place.

Every wait inside a kernel has a limit, after which the kernel returns with results that are not valid.  Calls do not wait for their kernels
and so cannot say so: ``binding.strassen_device_status()`` waits for the device and raises ``StrassenError`` if it has happened.
"""
from __future__ import annotations

import torch
from torch.autograd import forward_ad
from torch.autograd.graph import increment_version

from . import binding

__all__ = ["quant_rows", "rms_norm_quant", "silu_mul_quant", "route_experts", "W4Matrix", "W4Experts", "FeedForward", "ExpertsFeedForward"]

E4M3 = torch.float8_e4m3fn
_TYPES = {torch.bfloat16: binding.STRASSEN_BF16, torch.float16: binding.STRASSEN_F16, torch.float32: binding.STRASSEN_F32,
          E4M3: binding.STRASSEN_E4M3}
_ROW_TYPES = {t: _TYPES[t] for t in (torch.bfloat16, torch.float16, torch.float32)}
_X_TYPES = {t: _TYPES[t] for t in (torch.bfloat16, torch.float16, E4M3)}
_OUT_TYPES = {t: _TYPES[t] for t in (torch.bfloat16, torch.float16)}
_SCORES = {"softmax": binding.STRASSEN_SOFTMAX, "sigmoid": binding.STRASSEN_SIGMOID}

# Marks tensors as modified in place.  The public function looks at its argument's type first, which takes as long again.
_written = getattr(torch._C, "_increment_version", None) or increment_version

# The current device.  The public function looks first whether CUDA has been set up, which the tensors of a call show.
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device

# The current stream's handle by device index.  The public way there makes a Stream object first, which costs as much as a launch.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _gradients_off(name):
    """For a tensor that requires grad: its gradient is not dropped without a word."""
    if torch.is_grad_enabled():
        raise ValueError("%s requires grad, and the operators have no backward pass: detach it, or call them under torch.no_grad()" % name)


def _forward_mode():
    """Whether tensors may have tangents: within ``forward_ad.dual_level()``."""
    return getattr(forward_ad, "_current_level", 0) >= 0


def _tangents_off(**tensors):
    """Of the tensors of a call in forward mode: no tangent is dropped without a word."""
    for name, t in tensors.items():
        for part in t if isinstance(t, (tuple, list)) else (t,):
            if part is not None and forward_ad.unpack_dual(part).tangent is not None:
                raise ValueError("%s has a tangent, and the operators have no forward-mode derivative: use forward_ad.unpack_dual(t).primal" % name)


def _rows(name, t, shape, dtype, index):
    """Distance between the rows of ``t`` after checking it: the kernels index by the sizes alone, so a smaller tensor would be read or
    written out of bounds on the device."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == index:
        if t.requires_grad:
            _gradients_off(name)
        ld, step = t.stride()
        if step == 1 or shape[1] == 1:
            return ld
        raise ValueError("the rows of %s must be contiguous (last stride 1)" % name)
    if t.get_device() != index:
        raise ValueError("%s must be a tensor on cuda:%d, not on %s" % (name, index, t.device))
    if t.dtype != dtype:
        raise ValueError("%s must be %s, not %s" % (name, dtype, t.dtype))
    raise ValueError("%s has shape %s; %s is needed" % (name, tuple(t.shape), tuple(shape)))


def _packed(name, t, shape, dtype, index):
    """Address of ``t`` after checking it: contiguous."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s on cuda:%d, not %s %s on %s"
                         % (name, dtype, tuple(shape), index, t.dtype, tuple(t.shape), t.device))
    if t.requires_grad:
        _gradients_off(name)
    return t.data_ptr()


def _first(name, x, types):
    """(shape, type code, device index) of the tensor that the others have to go with."""
    kind = types.get(x.dtype)
    index = x.get_device()
    shape = x.shape
    if kind is None or index < 0 or len(shape) != 2:
        raise ValueError("%s must be a 2-D CUDA tensor of one of %s, not %s %s on %s"
                         % (name, ", ".join(str(t) for t in types), x.dtype, tuple(shape), x.device))
    return shape, kind, index


def _call(index, function, *args):
    """function(*args, stream) on the device's current stream, whose handle is returned."""
    stream = _raw_stream(index)
    if index == _current_device():
        function(*args, stream)
    else:
        with torch.cuda.device(index):
            function(*args, stream)
    return stream


def quant_rows(m, k, device="cuda"):
    """(q, scale): memory for m rows of k e4m3 values and their scales.  Rows start 16 bytes apart or a multiple of it, so that odd
    lengths keep the wide accesses."""
    ld = (int(k) + 15) // 16 * 16
    return torch.empty(int(m), ld, dtype=E4M3, device=device)[:, :int(k)], torch.empty(int(m), dtype=torch.float32, device=device)


def rms_norm_quant(x, weight, eps=1e-6, residual=None, out=None):
    """Root-mean-square norm of the rows of ``x`` (+ ``residual``) times ``weight``, in 8 bits.

    Returns (q, scale), or (q, scale, sum) with a residual: v ~ q * scale[:, None], sum = x + residual in x's type.  ``out`` is such a tuple to
    write to; its sum may be ``x`` or ``residual`` itself (the residual stream updated in place)."""
    if _forward_mode():
        _tangents_off(x=x, weight=weight, residual=residual, out=out)
    shape, kind, index = _first("x", x, _ROW_TYPES)
    m, k = shape
    dtype, given = x.dtype, out
    if out is None:
        out = quant_rows(m, k, x.device)
        if residual is not None:
            out += (torch.empty(m, k, dtype=dtype, device=x.device),)
    if len(out) != (2 if residual is None else 3):
        raise ValueError("out must be (q, scale), or (q, scale, sum) with a residual")
    q = out[0]
    ldx, ldq = _rows("x", x, shape, dtype, index), _rows("q", q, shape, E4M3, index)
    r = ldr = h = ldh = 0
    if residual is not None:
        ldr, ldh = _rows("residual", residual, shape, dtype, index), _rows("sum", out[2], shape, dtype, index)
        r, h = residual.data_ptr(), out[2].data_ptr()
    w, s = _packed("weight", weight, (k,), dtype, index), _packed("scale", out[1], (m,), torch.float32, index)
    _call(index, binding.strassen_rms_norm_quant, m, k, kind, x.data_ptr(), ldx, r, ldr, w, eps, h, ldh, q.data_ptr(), ldq, s)
    if given is not None:
        _written(out)
    return out


def silu_mul_quant(gate, up, out=None):
    """silu(gate) * up in 8 bits: (q, scale).  gate and up may be the halves of one tensor."""
    if _forward_mode():
        _tangents_off(gate=gate, up=up, out=out)
    shape, kind, index = _first("gate", gate, _ROW_TYPES)
    m, k = shape
    dtype, given = gate.dtype, out
    if out is None:
        out = quant_rows(m, k, gate.device)
    q = out[0]
    ldg, ldu, ldq = _rows("gate", gate, shape, dtype, index), _rows("up", up, shape, dtype, index), _rows("q", q, shape, E4M3, index)
    s = _packed("scale", out[1], (m,), torch.float32, index)
    _call(index, binding.strassen_silu_mul_quant, m, k, kind, gate.data_ptr(), ldg, up.data_ptr(), ldu, q.data_ptr(), ldq, s)
    if given is not None:
        _written(out)
    return out


def route_experts(logits, top, score="softmax", bias=None, groups=1, top_groups=1, renormalize=True, factor=1.0, out=None):
    """The ``top`` experts of each row of ``logits`` (tokens x experts) and their weights: (ids int32, weights float32), both tokens x top.

    ``score``: "softmax" or "sigmoid"; ``bias`` (float32, one per expert) is added to the scores for the choice alone; with ``groups`` only the
    experts of the ``top_groups`` best groups can be chosen.  Logits of -inf leave an expert out; ids are -1, with weight 0, where too few are left."""
    if _forward_mode():
        _tangents_off(logits=logits, bias=bias, out=out)
    shape, kind, index = _first("logits", logits, _ROW_TYPES)
    tokens, experts = shape
    given = out
    if score not in _SCORES:
        raise ValueError("score must be one of %s, not %r" % (", ".join(sorted(_SCORES)), score))
    if out is None:
        out = (torch.empty(tokens, top, dtype=torch.int32, device=logits.device), torch.empty(tokens, top, dtype=torch.float32, device=logits.device))
    ld = _rows("logits", logits, shape, logits.dtype, index)
    i, w = _packed("ids", out[0], (tokens, top), torch.int32, index), _packed("weights", out[1], (tokens, top), torch.float32, index)
    b = 0 if bias is None else _packed("bias", bias, (experts,), torch.float32, index)
    _call(index, binding.strassen_route_experts, tokens, experts, kind, logits.data_ptr(), ld, b, _SCORES[score], groups, top_groups, top, renormalize, factor, i, w)
    if given is not None:
        _written(out)
    return out


class _W4:
    """Laid-out 4-bit weights: one matrix or several of one size."""

    def __init__(self, q, scales, zeros, k, group, experts):
        self._h = None
        if _forward_mode():
            _tangents_off(scales=scales)
        if q.dtype != torch.uint8 or not q.is_cuda:
            raise ValueError("q must be a CUDA uint8 tensor, not %s on %s" % (q.dtype, q.device))
        if scales.dtype not in _OUT_TYPES:
            raise ValueError("scales must be bfloat16 or float16, not %s" % scales.dtype)
        self.n, self.k, self.group = int(q.shape[-2]), int(2 * q.shape[-1] if k is None else k), int(group)
        self.device, self._index = q.device, q.get_device()
        kind = _TYPES[scales.dtype]
        h = binding.strassen_w4_create(self.n, self.k, self.group, kind, zeros is not None) if experts is None else \
            binding.strassen_w4_create_experts(experts, self.n, self.k, self.group, kind, zeros is not None)
        self._h = h
        rows = self.n if experts is None else experts * self.n
        groups = (rows, (self.k + self.group - 1) // self.group)
        ldq = _rows("q", q.flatten(0, -2), (rows, (self.k + 1) // 2), torch.uint8, self._index)
        lds = _rows("scales", scales.flatten(0, -2), groups, scales.dtype, self._index)
        ldz = _rows("zeros", zeros.flatten(0, -2), groups, torch.uint8, self._index) if zeros is not None else 0
        q, scales, zeros = q.flatten(0, -2), scales.flatten(0, -2), zeros.flatten(0, -2) if zeros is not None else None
        self._packed = torch.empty(binding.strassen_w4_bytes(h), dtype=torch.uint8, device=self.device)
        self._stream = _call(self._index, binding.strassen_w4_pack, h, q.data_ptr(), ldq, scales.data_ptr(), lds, zeros.data_ptr() if zeros is not None else 0,
                             ldz, self._packed.data_ptr())
        self._others = set()             # handles of the other streams that products were enqueued on
        torch.cuda.current_stream(self.device).synchronize()

    @property
    def handle(self):
        return self._h

    @property
    def nbytes(self):
        """Device memory of the laid-out weights."""
        return self._packed.numel()

    def _output(self, x, rows, out, dtype):
        """(out, its type code, distance of its rows): new if None."""
        if out is None:
            if dtype is None:
                dtype = torch.bfloat16 if x.dtype == E4M3 else x.dtype
            out = torch.empty(rows, self.n, dtype=dtype, device=self.device)
        elif dtype is not None and out.dtype != dtype:
            raise ValueError("out is %s, dtype %s" % (out.dtype, dtype))
        kind = _OUT_TYPES.get(out.dtype)
        if kind is None:
            raise ValueError("the result is bfloat16 or float16, not %s" % out.dtype)
        return out, kind, _rows("out", out, (rows, self.n), out.dtype, self._index)

    def _workspace(self, need):
        # from the allocator of the current stream, which the call is enqueued on: free again when the call is done
        return torch.empty(need, dtype=torch.uint8, device=self.device)

    def close(self):
        """Free the weights.  Products may still be in flight: torch's allocator hands the memory out again when the streams that they
        were enqueued on have passed this point.  Nothing is waited for, so a matrix may also be collected while a graph is being captured."""
        if self._h is not None:
            h, self._h = self._h, None
            binding.strassen_w4_destroy(h)
            if getattr(self, "_packed", None) is not None:
                for stream in getattr(self, "_others", ()):
                    self._packed.record_stream(torch.cuda.ExternalStream(stream, self.device))
            self._packed = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class W4Matrix(_W4):
    """An n x k matrix held in 4 bits with a scale, and if wanted a zero point, for every ``group`` positions of a row:
    W = scale * (q - zero), zero 8 where none are given.

    ``q``: uint8 (n, ceil(k / 2)), two positions a byte, the first in the low half; ``scales``: bfloat16 or float16 (n, ceil(k / group));
    ``zeros``: uint8 of the same shape, 0..15.  They are laid out once into memory of the matrix's own and not referred to afterwards;
    the constructor waits for that, so the matrix can be used on any stream that lives as long as it does.  A captured graph does not
    keep it alive.
    """

    def __init__(self, q, scales, zeros=None, k=None, group=128):
        self._h = None
        if q.dim() != 2 or scales.dim() != 2 or (zeros is not None and zeros.dim() != 2):
            raise ValueError("q, scales and zeros must have 2 dimensions")
        super().__init__(q, scales, zeros, k, group, None)

    def __call__(self, x, x_scale=None, out=None, dtype=None):
        """x @ W.T (m x n) for rows ``x`` (m x k) in bfloat16, float16 or float8_e4m3fn, times ``x_scale`` (m floats: the scales of 8-bit rows).
        ``dtype``: of the result, bfloat16 or float16; x's own where it has 16 bits, else bfloat16.

        Up to 16 rows no weight is rounded, and a row's result does not depend on the rows beside it.  For more rows each weight is rounded once, to
        bfloat16 beside bfloat16 rows and to float16 beside the others."""
        if self._h is None:
            raise ValueError("the matrix has been closed")
        if _forward_mode():
            _tangents_off(x=x, x_scale=x_scale, out=out)
        shape, kind, index = _first("x", x, _X_TYPES)
        m, given = shape[0], out
        ldx = _rows("x", x, (m, self.k), x.dtype, self._index)
        out, out_kind, ldo = self._output(x, m, out, dtype)
        xs = 0 if x_scale is None else _packed("x_scale", x_scale, (m,), torch.float32, index)
        at, ws, need = x.data_ptr(), 0, 0
        # rows in 16 bits that start at multiples of 16 bytes need no workspace: not asked for them, a call in itself
        if m > binding.STRASSEN_W4_THIN_ROWS and (kind == binding.STRASSEN_E4M3 or at % 16 or ldx % 8):
            need = binding.strassen_w4_workspace_bytes(self._h, m, kind, at, ldx)
            if need:
                workspace = self._workspace(need)
                ws = workspace.data_ptr()
        stream = _call(index, binding.strassen_w4_matmul, self._h, m, kind, at, ldx, xs, out_kind, out.data_ptr(), ldo, ws, need)
        if stream != self._stream:
            self._others.add(stream)
        if given is not None:
            _written((out,))
        return out


class W4Experts(_W4):
    """The matrices of experts, all n x k, held as ``W4Matrix`` holds one: ``q`` (experts, n, ceil(k / 2)), ``scales`` and ``zeros``
    (experts, n, ceil(k / group))."""

    def __init__(self, q, scales, zeros=None, k=None, group=128):
        self._h = None
        if q.dim() != 3 or scales.dim() != 3 or (zeros is not None and zeros.dim() != 3):
            raise ValueError("q, scales and zeros must have 3 dimensions")
        for t in (q, scales) + (() if zeros is None else (zeros,)):
            if t.shape[0] != q.shape[0] or t.shape[1] != q.shape[1]:
                raise ValueError("q, scales and zeros must agree in their first two dimensions")
            if t.shape[0] > 1 and t.shape[1] > 1 and t.stride(0) != t.shape[1] * t.stride(1):
                raise ValueError("the matrices of experts must lie one after another, their rows at one distance")
        self.experts = int(q.shape[0])
        super().__init__(q, scales, zeros, k, group, self.experts)

    def __call__(self, x, ids, x_scale=None, weights=None, out=None, dtype=None):
        """Products of rows with the matrices that ``ids`` (int32, tokens x top, as ``route_experts`` gives them) name.

        ``x`` has a row for each token, or one for each id (row token * top + j).  Without ``weights`` the result has a row for each id; with
        ``weights`` (float32, tokens x top) one for each token: the weighted sum of its ids' rows.  Ids outside 0 .. experts - 1 are no expert.
        Weights of the matrices are rounded as ``W4Matrix`` does it, beyond 32 ids."""
        if self._h is None:
            raise ValueError("the matrices have been closed")
        if _forward_mode():
            _tangents_off(x=x, x_scale=x_scale, weights=weights, out=out)
        shape, kind, index = _first("x", x, _X_TYPES)
        if len(ids.shape) != 2:
            raise ValueError("ids must be tokens x top, not %s" % (tuple(ids.shape),))
        tokens, top = ids.shape
        rows, given = shape[0], out
        if rows != tokens and rows != tokens * top:
            raise ValueError("x has %d rows; %d (one for each token) or %d (one for each id) are needed" % (rows, tokens, tokens * top))
        ldx, i = _rows("x", x, (rows, self.k), x.dtype, self._index), _packed("ids", ids, (tokens, top), torch.int32, index)
        out, out_kind, ldo = self._output(x, tokens if weights is not None else tokens * top, out, dtype)
        xs = 0 if x_scale is None else _packed("x_scale", x_scale, (rows,), torch.float32, index)
        w = 0 if weights is None else _packed("weights", weights, (tokens, top), torch.float32, index)
        ws = need = 0
        if tokens * top > binding.STRASSEN_W4_THIN_IDS:
            need = binding.strassen_w4_experts_workspace_bytes(self._h, tokens, top, weights is not None)
            workspace = self._workspace(need)
            ws = workspace.data_ptr()
        stream = _call(index, binding.strassen_w4_experts, self._h, tokens, top, i, kind, x.data_ptr(), ldx, rows != tokens, xs, w, out_kind, out.data_ptr(), ldo, ws, need)
        if stream != self._stream:
            self._others.add(stream)
        if given is not None:
            _written((out,))
        return out


class FeedForward:
    """One served feed-forward block:  h = x + residual;  y = down(silu(gate(n)) * up(n)) with n the norm of h.

    ``gate_up`` is a W4Matrix of 2 f rows (gate above up) over the model's width, ``down`` one of the width's rows over f."""

    def __init__(self, norm_weight, gate_up, down, eps=1e-6):
        _check_block(norm_weight, gate_up, down)
        self.norm_weight, self.gate_up, self.down, self.eps = norm_weight, gate_up, down, eps

    def __call__(self, x, residual):
        """(y, h), both of x's type: the block's output, to be added to the residual stream h by the next norm.  Beside float32 rows the products
        give bfloat16, and y holds its values."""
        q, s, h = rms_norm_quant(x, self.norm_weight, self.eps, residual=residual)
        gu = self.gate_up(q, s, dtype=x.dtype if x.dtype is not torch.float32 else None)
        f = self.down.k
        q, s = silu_mul_quant(gu[:, :f], gu[:, f:])
        return self.down(q, s, dtype=gu.dtype).to(x.dtype), h


class ExpertsFeedForward:
    """The same with experts: ``gate_up`` and ``down`` are W4Experts; further arguments are those of ``route_experts``.

    ``router`` gives the logits.  As a matrix (experts x width, of x's type) it is multiplied, in 32 bits by torch, by the norm's 8-bit rows, which is
    what the experts see; their three bits of fraction decide between experts that are close, so that some tokens go to other experts than the unrounded norm
    would send them to.  A router that was trained on the norm in more bits is given as a function of the residual stream h, which returns the logits
    (rows x experts): ``lambda h: torch.nn.functional.rms_norm(h, (width,), norm_weight, eps) @ matrix.t()``."""

    def __init__(self, norm_weight, router, gate_up, down, top, eps=1e-6, **routing):
        _check_block(norm_weight, gate_up, down)
        if gate_up.experts != down.experts:
            raise ValueError("%d and %d experts" % (gate_up.experts, down.experts))
        if not callable(router) and tuple(router.shape) != (gate_up.experts, gate_up.k):
            raise ValueError("%d experts of width %d, and a router %s" % (gate_up.experts, gate_up.k, tuple(router.shape)))
        self.norm_weight, self.router, self.gate_up, self.down, self.top, self.eps, self.routing = norm_weight, router, gate_up, down, top, eps, routing

    def __call__(self, x, residual):
        """(y, h), as FeedForward."""
        q, s, h = rms_norm_quant(x, self.norm_weight, self.eps, residual=residual)
        if callable(self.router):
            logits = self.router(h)
            if tuple(logits.shape) != (x.shape[0], self.gate_up.experts):
                raise ValueError("the router gave logits of shape %s for %d rows and %d experts" % (tuple(logits.shape), x.shape[0], self.gate_up.experts))
        else:
            logits = (q.to(torch.float32) * s[:, None]) @ self.router.float().t()
        ids, weights = route_experts(logits, self.top, **self.routing)
        gu = self.gate_up(q, ids, s, dtype=x.dtype if x.dtype is not torch.float32 else None)
        f = self.down.k
        q, s = silu_mul_quant(gu[:, :f], gu[:, f:])
        return self.down(q, ids, s, weights=weights, dtype=gu.dtype).to(x.dtype), h


def _check_block(norm_weight, gate_up, down):
    if gate_up.n != 2 * down.k or gate_up.k != down.n or tuple(norm_weight.shape) != (gate_up.k,):
        raise ValueError("a block of width %d needs a norm of that size, gate_up (2 f x %d) and down (%d x f); got %s, %d x %d and %d x %d"
                         % (gate_up.k, gate_up.k, gate_up.k, tuple(norm_weight.shape), gate_up.n, gate_up.k, down.n, down.k))


def quantize_w4(w, group=128, dtype=torch.bfloat16):
    """(q, scales, zeros) of a float matrix by rounding between each group's smallest and largest value (torch operations: for examples and
    tests, not for a served path)."""
    n, k = w.shape
    groups = (k + group - 1) // group
    v = torch.nn.functional.pad(w.float(), (0, groups * group - k)).view(n, groups, group)
    lo, hi = v.amin(-1).clamp_max(0.0), v.amax(-1).clamp_min(0.0)
    scales = ((hi - lo) / 15).clamp_min(1e-6).to(dtype)
    zeros = (-lo / scales.float()).round().clamp(0, 15)
    q = ((v / scales.float()[..., None]).round() + zeros[..., None]).clamp(0, 15).to(torch.uint8).view(n, -1)[:, :k]
    q = torch.nn.functional.pad(q, (0, k % 2))
    return (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous(), scales, zeros.to(torch.uint8)


def main():
    """A block of width 4096 with 16384 inner features: one token and a prompt, against the same block in 32 bits."""
    width, inner, group = 4096, 16384, 128
    g = torch.Generator("cuda").manual_seed(0)
    weights, plain = [], []
    for n, k in ((2 * inner, width), (width, inner)):
        q, s, z = quantize_w4(torch.randn(n, k, device="cuda", generator=g) * 0.02, group)
        weights.append(W4Matrix(q, s, z, k=k, group=group))
        nibbles = torch.stack([q & 15, q >> 4], -1).view(n, k).float()
        plain.append(s.float().repeat_interleave(group, 1) * (nibbles - z.float().repeat_interleave(group, 1)))
    norm = torch.ones(width, device="cuda", dtype=torch.bfloat16)
    block = FeedForward(norm, *weights)
    for m in (1, 512):
        x, r = (torch.randn(m, width, device="cuda", generator=g).bfloat16() for _ in range(2))
        y, h = block(x, r)
        n = x.float() + r.float()
        n = n * (n.square().mean(-1, keepdim=True) + block.eps).rsqrt()
        gu = n @ plain[0].t()
        want = (torch.nn.functional.silu(gu[:, :inner]) * gu[:, inner:]) @ plain[1].t()
        start, stop = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for _ in range(3):
            block(x, r)
        start.record()
        for _ in range(20):
            block(x, r)
        stop.record()
        torch.cuda.synchronize()
        print("%4d rows: %7.1f us a block, %.3f of the 32-bit block's output is the rounding to 8 bits"
              % (m, start.elapsed_time(stop) / 20 * 1e3, float((y.float() - want).norm() / want.norm())))


if __name__ == "__main__":
    main()
