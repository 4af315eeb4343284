"""Feed-forward operators of a served model on torch tensors: rows of activations in 8 bits, weights in 4.

The work is done by the kernels behind ``strassen_rms_norm_quant``, ``strassen_silu_mul_quant`` and ``strassen_w4_matmul``
(``include/strassen_b200.h`` has their formulas); here are the checks of shapes, types and devices, the memory and the
current stream.  ``FeedForward`` runs them together as one block; ``python -m paper_1202_3173_b200.feed_forward`` tries it out.

Rows are 2-D CUDA tensors whose last dimension is contiguous; rows may be any distance apart (views of wider tensors).  Calls are
enqueued on the current stream, allocate nothing when ``out`` is given, and can be captured into a CUDA graph.
"""
from __future__ import annotations

import torch

from . import binding

__all__ = ["quant_rows", "rms_norm_quant", "silu_mul_quant", "W4Matrix", "FeedForward"]

E4M3 = torch.float8_e4m3fn
_TYPES = {torch.bfloat16: binding.STRASSEN_BF16, torch.float16: binding.STRASSEN_F16, torch.float32: binding.STRASSEN_F32,
          E4M3: binding.STRASSEN_E4M3}
_ROW_TYPES = (torch.bfloat16, torch.float16, torch.float32)


def _rows(name, t, shape, dtype, device):
    """Distance between the rows of ``t`` after checking it: the kernels index by the sizes alone, so a smaller tensor would be read or
    written out of bounds on the device."""
    if t.dtype is not dtype or t.shape != shape or t.device != device or not t.is_cuda or (t.stride(1) != 1 and shape[1] > 1):
        if not t.is_cuda or t.device != device:
            raise ValueError("%s must be a CUDA tensor on %s, not on %s" % (name, device, t.device))
        if t.dtype != dtype:
            raise ValueError("%s must be %s, not %s" % (name, dtype, t.dtype))
        if tuple(t.shape) != tuple(shape):
            raise ValueError("%s has shape %s; %s is needed" % (name, tuple(t.shape), tuple(shape)))
        raise ValueError("the rows of %s must be contiguous (last stride 1)" % name)
    return t.stride(0)


def _vector(name, t, size, dtype, device):
    if t.dtype is not dtype or t.shape != (size,) or t.device != device or (t.stride(0) != 1 and size > 1):
        raise ValueError("%s must be a contiguous %s vector of %d elements on %s, not %s %s on %s"
                         % (name, dtype, size, device, t.dtype, tuple(t.shape), t.device))
    return t.data_ptr()


def _first(name, x, types):
    if x.dim() != 2 or not x.is_cuda or x.dtype not in types:
        raise ValueError("%s must be a 2-D CUDA tensor of one of %s, not %s %s on %s"
                         % (name, ", ".join(str(t) for t in types), x.dtype, tuple(x.shape), x.device))


def _call(device, function, *args):
    """function(*args, stream) on the device's current stream."""
    if device.index == torch.cuda.current_device():
        function(*args, torch.cuda.current_stream().cuda_stream)
    else:
        with torch.cuda.device(device):
            function(*args, torch.cuda.current_stream().cuda_stream)


def quant_rows(m, k, device="cuda"):
    """(q, scale): memory for m rows of k e4m3 values and their scales.  Rows start 16 bytes apart or a multiple of it, so that odd
    lengths keep the wide accesses."""
    ld = (int(k) + 15) // 16 * 16
    return torch.empty(int(m), ld, dtype=E4M3, device=device)[:, :int(k)], torch.empty(int(m), dtype=torch.float32, device=device)


def rms_norm_quant(x, weight, eps=1e-6, residual=None, out=None):
    """Root-mean-square norm of the rows of ``x`` (+ ``residual``) times ``weight``, in 8 bits.

    Returns (q, scale), or (q, scale, sum) with a residual: v ~ q * scale[:, None], sum = x + residual in x's type.  ``out`` is such a tuple to
    write to; its sum may be ``x`` or ``residual`` itself (the residual stream updated in place)."""
    _first("x", x, _ROW_TYPES)
    m, k = shape = x.shape
    device, dtype = x.device, x.dtype
    if out is None:
        out = quant_rows(m, k, device)
        if residual is not None:
            out += (torch.empty(m, k, dtype=dtype, device=device),)
    if len(out) != (2 if residual is None else 3):
        raise ValueError("out must be (q, scale), or (q, scale, sum) with a residual")
    ldx, ldq = _rows("x", x, shape, dtype, device), _rows("q", out[0], shape, E4M3, device)
    r = ldr = h = ldh = 0
    if residual is not None:
        ldr, ldh = _rows("residual", residual, shape, dtype, device), _rows("sum", out[2], shape, dtype, device)
        r, h = residual.data_ptr(), out[2].data_ptr()
    w, s = _vector("weight", weight, k, dtype, device), _vector("scale", out[1], m, torch.float32, device)
    _call(device, binding.strassen_rms_norm_quant, m, k, _TYPES[dtype], x.data_ptr(), ldx, r, ldr, w, eps, h, ldh, out[0].data_ptr(), ldq, s)
    return out


def silu_mul_quant(gate, up, out=None):
    """silu(gate) * up in 8 bits: (q, scale).  gate and up may be the halves of one tensor."""
    _first("gate", gate, _ROW_TYPES)
    m, k = shape = gate.shape
    device, dtype = gate.device, gate.dtype
    if out is None:
        out = quant_rows(m, k, device)
    ldg, ldu = _rows("gate", gate, shape, dtype, device), _rows("up", up, shape, dtype, device)
    ldq, s = _rows("q", out[0], shape, E4M3, device), _vector("scale", out[1], m, torch.float32, device)
    _call(device, binding.strassen_silu_mul_quant, m, k, _TYPES[dtype], gate.data_ptr(), ldg, up.data_ptr(), ldu, out[0].data_ptr(), ldq, s)
    return out


class W4Matrix:
    """An n x k matrix held in 4 bits with a scale, and if wanted a zero point, for every ``group`` positions of a row:
    W = scale * (q - zero), zero 8 where none are given.

    ``q``: uint8 (n, ceil(k / 2)), two positions a byte, the first in the low half; ``scales``: bfloat16 or float16 (n, ceil(k / group));
    ``zeros``: uint8 of the same shape, 0..15.  They are laid out once into memory of the matrix's own and not referred to afterwards;
    the constructor waits for that, so the matrix can be used on any stream.
    """

    def __init__(self, q, scales, zeros=None, k=None, group=128):
        self._h = None
        if q.dim() != 2 or q.dtype != torch.uint8 or not q.is_cuda:
            raise ValueError("q must be a 2-D CUDA uint8 tensor, not %s %s on %s" % (q.dtype, tuple(q.shape), q.device))
        if scales.dtype not in (torch.bfloat16, torch.float16):
            raise ValueError("scales must be bfloat16 or float16, not %s" % scales.dtype)
        self.n, self.k, self.group = int(q.shape[0]), int(2 * q.shape[1] if k is None else k), int(group)
        self.device = q.device
        h = binding.strassen_w4_create(self.n, self.k, self.group, _TYPES[scales.dtype], zeros is not None)
        self._h = h
        groups = (self.n, (self.k + self.group - 1) // self.group)
        ldq = _rows("q", q, (self.n, (self.k + 1) // 2), torch.uint8, self.device)
        lds = _rows("scales", scales, groups, scales.dtype, self.device)
        ldz = _rows("zeros", zeros, groups, torch.uint8, self.device) if zeros is not None else 0
        self._packed = torch.empty(binding.strassen_w4_bytes(h), dtype=torch.uint8, device=self.device)
        _call(self.device, binding.strassen_w4_pack, h, q.data_ptr(), ldq, scales.data_ptr(), lds, zeros.data_ptr() if zeros is not None else 0,
              ldz, self._packed.data_ptr())
        torch.cuda.current_stream(self.device).synchronize()

    @property
    def handle(self):
        return self._h

    @property
    def nbytes(self):
        """Device memory of the laid-out matrix."""
        return self._packed.numel()

    def __call__(self, x, x_scale=None, out=None, dtype=None):
        """x @ W.T (m x n) for rows ``x`` (m x k) in bfloat16, float16 or float8_e4m3fn, times ``x_scale`` (m floats: the scales of 8-bit rows).
        ``dtype``: of the result, bfloat16 or float16; x's own where it has 16 bits, else bfloat16."""
        if self._h is None:
            raise ValueError("the matrix has been closed")
        _first("x", x, (torch.bfloat16, torch.float16, E4M3))
        m, device = x.shape[0], self.device
        if out is None:
            if dtype is None:
                dtype = torch.bfloat16 if x.dtype == E4M3 else x.dtype
            out = torch.empty(m, self.n, dtype=dtype, device=device)
        elif dtype is not None and out.dtype != dtype:
            raise ValueError("out is %s, dtype %s" % (out.dtype, dtype))
        if out.dtype is not torch.bfloat16 and out.dtype is not torch.float16:
            raise ValueError("the result is bfloat16 or float16, not %s" % out.dtype)
        ldx, ldo = _rows("x", x, (m, self.k), x.dtype, device), _rows("out", out, (m, self.n), out.dtype, device)
        xs = 0 if x_scale is None else _vector("x_scale", x_scale, m, torch.float32, device)
        at, kind, ws, need = x.data_ptr(), _TYPES[x.dtype], 0, 0
        if m > binding.STRASSEN_W4_THIN_ROWS:
            need = binding.strassen_w4_workspace_bytes(self._h, m, kind, at, ldx)
            if need:
                workspace = torch.empty(need, dtype=torch.uint8, device=device)      # of the current stream, like the call
                ws = workspace.data_ptr()
        _call(device, binding.strassen_w4_matmul, self._h, m, kind, at, ldx, xs, _TYPES[out.dtype], out.data_ptr(), ldo, ws, need)
        return out

    def close(self):
        """Free the matrix.  Products may still be in flight on any stream, so its device is synchronised first."""
        if self._h is not None:
            if getattr(self, "_packed", None) is not None:
                torch.cuda.synchronize(self.device)
            binding.strassen_w4_destroy(self._h)
            self._h = self._packed = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class FeedForward:
    """One served feed-forward block:  h = x + residual;  y = down(silu(gate(n)) * up(n)) with n the norm of h.

    ``gate_up`` is a W4Matrix of 2 f rows (gate above up) over the model's width, ``down`` one of the width's rows over f."""

    def __init__(self, norm_weight, gate_up, down, eps=1e-6):
        if gate_up.n != 2 * down.k or gate_up.k != down.n or tuple(norm_weight.shape) != (gate_up.k,):
            raise ValueError("a block of width %d needs a norm of that size, gate_up (2 f x %d) and down (%d x f); got %s, %d x %d and %d x %d"
                             % (gate_up.k, gate_up.k, gate_up.k, tuple(norm_weight.shape), gate_up.n, gate_up.k, down.n, down.k))
        self.norm_weight, self.gate_up, self.down, self.eps = norm_weight, gate_up, down, eps

    def __call__(self, x, residual):
        """(y, h): the block's output, to be added to the residual stream h by the next norm."""
        q, s, h = rms_norm_quant(x, self.norm_weight, self.eps, residual=residual)
        gu = self.gate_up(q, s, dtype=x.dtype if x.dtype is not torch.float32 else None)
        f = self.down.k
        q, s = silu_mul_quant(gu[:, :f], gu[:, f:])
        return self.down(q, s, dtype=gu.dtype), h


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
