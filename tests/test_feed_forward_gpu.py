"""The feed-forward operators against their formulas in 64 bits: norm and gate with 8-bit rows, products with 4-bit weights.

Tolerances.  u is the unit roundoff of a format: 2^-4 for e4m3 (smallest step of its subnormals 2^-9), 2^-8 for bf16, 2^-11 for f16.
  8-bit rows   |q s - v| <= 2^-4 |v| + 2^-10 s + 1e-5 max|v|   (one rounding of v / s; the last term: sums and quotients in 32 bits)
               |s - s64| <= 1e-5 s64, sum equal to the sum in 32 bits rounded once
  products     |y - y64| <= u |y64| + (K 2^-23 + w) sum_k |x_k| |S| (|Q - Z| + Z) xs
               u for the result's rounding, K 2^-23 for sums in 32 bits; w = 0 up to 16 rows, where no weight is rounded, and beyond
               that the unit roundoff of the 16-bit weights (bf16 for bf16 rows, f16 for f16 and e4m3 rows)
               and in the 2-norm over the result: at most 2 u + 2 w + K 2^-23 (roundings of independent signs do not add up)
"""
import pytest
import torch

from paper_1202_3173_b200 import StrassenError, binding

pytestmark = pytest.mark.gpu

BF16, F16, F32, E4M3 = torch.bfloat16, torch.float16, torch.float32, torch.float8_e4m3fn
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11}
EPS = 1e-6


def sw():
    import paper_1202_3173_b200 as m
    return m


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def strided(t, pad, shift=0, fill=float("nan")):
    """The values of t as rows of a wider buffer that starts ``shift`` elements in; what lies between is ``fill``."""
    m, k = t.shape
    buf = torch.full((m * (k + pad) + shift + pad,), fill, device=t.device).to(t.dtype)
    v = buf[shift:shift + m * (k + pad)].view(m, k + pad)[:, :k]
    v.copy_(t)
    return v


# ---- rows to 8 bits ----------------------------------------------------------------------------------------------

def check_rows(q, s, v):
    s64 = (v.abs().amax(1) / 448).clamp_min(2.0 ** -64)
    assert ((s.double() - s64).abs() <= 1e-5 * s64).all()
    got = q.double() * s.double()[:, None]
    lim = 2.0 ** -4 * v.abs() + 2.0 ** -10 * s64[:, None] + 1e-5 * v.abs().amax(1, keepdim=True)
    assert torch.isfinite(got).all() and ((got - v).abs() <= lim).all(), float(((got - v).abs() - lim).max())
    # the row's largest value takes the largest e4m3 number
    big = v.abs().amax(1) > 448 * 2.0 ** -64
    assert (q.float().abs().amax(1)[big] == 448).all()


def norm64(x, w, r=None):
    h = x.double() if r is None else x.double() + r.double()
    return h / torch.sqrt((h * h).mean(1, keepdim=True) + EPS) * w.double()


NORM_SHAPES = [(1, 1), (3, 7), (1, 8), (5, 64), (2, 1000), (7, 1023), (4, 4096), (3, 8200), (2, 12345), (1, 16384), (300, 512), (2, 40000), (2, 40001)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,k", NORM_SHAPES)
def test_norm(m, k, dtype):
    g = gen(m * 131 + k)
    x, r = (torch.randn(m, k, device="cuda", generator=g).to(dtype) * 3 for _ in range(2))
    w = (1 + 0.3 * torch.randn(k, device="cuda", generator=g)).to(dtype)
    q, s = sw().rms_norm_quant(x, w, EPS)
    check_rows(q, s, norm64(x, w))
    q, s, h = sw().rms_norm_quant(x, w, EPS, residual=r)
    check_rows(q, s, norm64(x, w, r))
    assert torch.equal(h, (x.float() + r.float()).to(dtype))


@pytest.mark.parametrize("pad,shift", [(8, 0), (8, 8), (1, 0), (3, 1), (16, 5)])
@pytest.mark.parametrize("k", [7, 256, 2049, 40001])
def test_norm_strides_and_alignment(k, pad, shift):
    g = gen(k + pad)
    x, r = (strided(torch.randn(5, k, device="cuda", generator=g).to(F16), pad, shift) for _ in range(2))
    w = torch.rand(k + shift, device="cuda", generator=g).to(F16)[shift:]
    buf = torch.zeros(5, k + pad + shift, device="cuda").to(E4M3)
    q, s, h = buf[:, shift:shift + k], torch.empty(5, device="cuda"), strided(torch.zeros(5, k, device="cuda").to(F16), pad, shift)
    got = sw().rms_norm_quant(x, w, EPS, residual=r, out=(q, s, h))
    assert got[0] is q and got[2] is h
    check_rows(q, s, norm64(x, w, r))
    assert torch.equal(h, (x.float() + r.float()).to(F16))
    # nothing was written beside the rows
    assert (buf[:, :shift].float() == 0).all() and (buf[:, shift + k:].float() == 0).all()
    wide = h.as_strided((4, pad), (k + pad, 1), h.storage_offset() + k)
    assert torch.isnan(wide.float()).all()


@pytest.mark.parametrize("k", [300, 4096, 70001])
def test_norm_sum_in_place(k):
    g = gen(k)
    for which in ("x", "residual"):
        x, r = (torch.randn(6, k, device="cuda", generator=g).to(BF16) for _ in range(2))
        want, v = (x.float() + r.float()).to(BF16), norm64(x, torch.ones(k, device="cuda"), r)
        q, s = sw().quant_rows(6, k)
        sw().rms_norm_quant(x, torch.ones(k, device="cuda", dtype=BF16), EPS, residual=r, out=(q, s, x if which == "x" else r))
        assert torch.equal(x if which == "x" else r, want)
        check_rows(q, s, v)


@pytest.mark.parametrize("pad,shift", [(0, 0), (7, 0), (1, 3), (8, 8)])
@pytest.mark.parametrize("k", [1, 7, 31, 64, 100, 128, 200, 256, 300, 511, 777, 1024, 1025, 2049, 4096, 6001, 8192, 12345, 16383, 16384])
def test_many_rows(k, pad, shift):
    """Rows enough for CTAs that stay and copy ahead: each alignment, the first and last row of the matrix included, sums in place too."""
    g = gen(k + pad)
    for dtype in (BF16, F16, F32):
        m = 700
        x, r = (strided(torch.randn(m, k, device="cuda", generator=g).to(dtype), pad, shift) for _ in range(2))
        w = (1 + 0.3 * torch.randn(k, device="cuda", generator=g)).to(dtype)
        q, s = sw().quant_rows(m, k)
        sw().rms_norm_quant(x, w, EPS, out=(q, s))
        check_rows(q, s, norm64(x, w))
        want, v = (x.float() + r.float()).to(dtype), norm64(x, w, r)
        total = torch.empty(m, k, device="cuda", dtype=dtype)
        sw().rms_norm_quant(x, w, EPS, residual=r, out=(q, s, total))
        check_rows(q, s, v)
        assert torch.equal(total, want)
        a, b = x.double(), r.double()
        sw().silu_mul_quant(x, r, out=(q, s))
        check_rows(q, s, a * torch.special.expit(a) * b)
        sw().rms_norm_quant(x, w, EPS, residual=r, out=(q, s, r))
        check_rows(q, s, v)
        assert torch.equal(r, want)
    binding.strassen_device_status()


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("pad,shift", [(0, 0), (7, 0), (1, 3)])
@pytest.mark.parametrize("k", [600, 1025, 2047, 2048, 4096, 4099, 8192, 12345, 16384])
def test_matrices_of_many_megabytes(k, pad, shift, dtype):
    """Norms with enough to do for CTAs that stay and copy ahead, each number of threads and pieces, sums staged or not and in place; gates of as much."""
    g = gen(k + pad)
    m = 90000000 // (k * dtype.itemsize)
    x, r = (strided(torch.randn(m, k, device="cuda", generator=g).to(dtype), pad, shift) for _ in range(2))
    w = (1 + 0.3 * torch.randn(k, device="cuda", generator=g)).to(dtype)
    q, s = sw().quant_rows(m, k)
    sw().rms_norm_quant(x, w, EPS, out=(q, s))
    check_rows(q, s, norm64(x, w))
    sw().silu_mul_quant(x, r, out=(q, s))
    check_rows(q, s, x.double() * torch.special.expit(x.double()) * r.double())
    want, v = (x.float() + r.float()).to(dtype), norm64(x, w, r)
    total = torch.empty(m, k, device="cuda", dtype=dtype)
    sw().rms_norm_quant(x, w, EPS, residual=r, out=(q, s, total))
    check_rows(q, s, v)
    assert torch.equal(total, want)
    sw().rms_norm_quant(x, w, EPS, residual=r, out=(q, s, r))
    check_rows(q, s, v)
    assert torch.equal(r, want)
    binding.strassen_device_status()


def test_norm_rows_of_zeros_nan_and_infinity():
    for k in (96, 40000):
        x = torch.randn(6, k, device="cuda")
        x[1] = 0
        x[2, 5] = float("nan")
        x[3, 7] = float("inf")
        x[4] = 1e-30                                  # far below eps: the smallest scale
        q, s = sw().rms_norm_quant(x, torch.ones(k, device="cuda"), EPS)
        assert s[1] == 2.0 ** -64 and (q[1].float() == 0).all()
        assert torch.isnan(s[2:4]).all() and torch.isnan(q[2:4].float()).all()
        check_rows(q[[0, 1, 4, 5]], s[[0, 1, 4, 5]], norm64(x[[0, 1, 4, 5]], torch.ones(k, device="cuda")))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("m,f", [(1, 1), (3, 7), (2, 64), (4, 1000), (33, 2047), (1, 16384), (5, 11008), (2, 33000), (2, 40001)])
def test_gate(m, f, dtype):
    g = gen(m + f)
    gu = torch.randn(m, 2 * f, device="cuda", generator=g).to(dtype) * 4
    q, s = sw().silu_mul_quant(gu[:, :f], gu[:, f:])
    a, b = gu.double().split(f, 1)
    check_rows(q, s, a * torch.special.expit(a) * b)


def test_gate_extremes():
    g = torch.tensor([[-100.0, -1e4, 0.0, 50.0], [0.0, 0.0, 0.0, 0.0], [float("nan"), 1.0, 1.0, 1.0], [1.0, 2.0, 3.0, 4.0]], device="cuda")
    u = torch.tensor([[3.0, 5.0, 7.0, -2.0], [1.0, 2.0, 3.0, 4.0], [1.0, 1.0, 1.0, 1.0], [0.0, 0.0, 0.0, 0.0]], device="cuda")
    q, s = sw().silu_mul_quant(g, u)
    check_rows(q[[0, 1, 3]], s[[0, 1, 3]], (g.double() * torch.special.expit(g.double()) * u.double())[[0, 1, 3]])
    assert (s[[1, 3]] == 2.0 ** -64).all() and torch.isnan(s[2]) and torch.isnan(q[2].float()).all()


def test_row_operators_take_no_rows():
    x = torch.empty(0, 64, device="cuda", dtype=BF16)
    q, s, h = sw().rms_norm_quant(x, torch.ones(64, device="cuda", dtype=BF16), EPS, residual=x)
    assert q.shape == (0, 64) and s.shape == (0,) and h.shape == (0, 64)
    assert sw().silu_mul_quant(x, x)[0].shape == (0, 64)


# ---- products with 4-bit weights -----------------------------------------------------------------------------------

def weights(n, k, group, zeros, dtype, seed, spread=1.0):
    g = gen(seed)
    groups = -(-k // group)
    q = torch.randint(0, 256, (n, (k + 1) // 2), device="cuda", generator=g, dtype=torch.uint8)
    s = (0.01 * torch.randn(n, groups, device="cuda", generator=g) * spread ** torch.rand(n, groups, device="cuda", generator=g)).to(dtype)
    z = torch.randint(0, 16, (n, groups), device="cuda", generator=g, dtype=torch.uint8) if zeros else None
    return q, s, z


def dense64(q, s, z, k, group):
    """(W, |S| (|Q - Z| + Z)) in 64 bits."""
    n = q.shape[0]
    nib = torch.empty(n, 2 * q.shape[1], device="cuda", dtype=torch.float64)
    nib[:, 0::2] = (q & 15).double()
    nib[:, 1::2] = (q >> 4).double()
    at = torch.arange(k, device="cuda") // group
    zz = z.double()[:, at] if z is not None else torch.full((n, k), 8.0, device="cuda", dtype=torch.float64)
    d = nib[:, :k] - zz
    return s.double()[:, at] * d, s.double()[:, at].abs() * (d.abs() + zz)


def rows(m, k, dtype, seed):
    g = gen(seed)
    x = torch.randn(m, k, device="cuda", generator=g)
    if dtype != E4M3:
        return x.to(dtype), None
    xs = x.abs().amax(1) / 448
    return (x / xs[:, None]).clamp(-448, 448).to(E4M3), xs


def check_product(y, x, xs, W, A, out_dtype):
    m, k = x.shape
    xd = x.double() if xs is None else x.double() * xs.double()[:, None]
    want, size = xd @ W.t(), xd.abs() @ A.t()
    w = 0.0 if m <= 16 else U[BF16] if x.dtype == BF16 else U[F16]
    assert y.dtype == out_dtype and torch.isfinite(y).all()
    err = (y.double() - want).abs()
    lim = U[out_dtype] * want.abs() + (k * 2.0 ** -23 + w) * size + (6e-8 if out_dtype == F16 else 0)      # f16 results below its normal range
    assert (err <= lim).all(), float((err - lim).max())
    assert err.norm() <= (2 * U[out_dtype] + 2 * w + k * 2.0 ** -23) * want.norm() + 6e-8 * err.numel() ** 0.5, float(err.norm() / want.norm())


W4_SHAPES = [(1, 1, 1), (1, 128, 128), (2, 16, 130), (1, 4096, 4096), (3, 100, 1000), (5, 129, 257), (8, 512, 2048), (9, 33, 640), (16, 300, 4097),
             (17, 256, 512), (31, 130, 300), (64, 1000, 1024), (100, 257, 4099), (129, 128, 384), (257, 640, 1111), (1, 40, 16384), (2, 5000, 96)]


@pytest.mark.parametrize("group,zeros", [(32, False), (32, True), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("m,n,k", W4_SHAPES)
def test_w4_product(m, n, k, group, zeros):
    products(m, n, k, group, zeros)


@pytest.mark.parametrize("m,n,k", [(3000, 4000, 100), (2100, 2600, 200), (1100, 5000, 300), (1300, 4200, 500), (700, 9000, 1500)])
def test_w4_product_of_more_tiles_than_the_gpu_holds(m, n, k):
    """Tiles of one, two and more steps of the inner dimension, taken by CTAs that stay."""
    products(m, n, k, 64, True)


def products(m, n, k, group, zeros):
    for dtype, out_dtype, sdtype in ((BF16, BF16, BF16), (F16, F16, F16), (E4M3, BF16, BF16), (E4M3, F16, F16), (BF16, F16, F16)):
        q, s, z = weights(n, k, group, zeros, sdtype, n + k)
        W, A = dense64(q, s, z, k, group)
        x, xs = rows(m, k, dtype, m + k)
        matrix = sw().W4Matrix(q, s, z, k=k, group=group)
        check_product(matrix(x, xs, dtype=out_dtype), x, xs, W, A, out_dtype)


@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (2, 0), (3, 1), (8, 0), (8, 8), (16, 16), (7, 3)])
@pytest.mark.parametrize("m", [1, 6, 20, 150])
def test_w4_strides_and_alignment(m, pad, shift):
    n, k, group = 200, 777, 64
    for dtype in (BF16, E4M3):
        q, s, z = weights(n, k, group, True, BF16, 5)
        W, A = dense64(q, s, z, k, group)
        x, xs = rows(m, k, dtype, 9)
        x = strided(x, pad, shift)                    # NaN beside the rows: none of it may reach a sum
        qs, ss, zs = strided(q, pad, shift, 0), strided(s, pad, shift), strided(z, pad, shift, 0)
        out = strided(torch.zeros(m, n, device="cuda").to(BF16), pad, shift, 7.0)
        matrix = sw().W4Matrix(qs, ss, zs, k=k, group=group)
        assert matrix(x, xs, out=out) is out
        check_product(out, x, xs, W, A, BF16)
        if m > 1 and pad:
            assert (out.as_strided((m - 1, pad), (n + pad, 1), out.storage_offset() + n) == 7).all()


@pytest.mark.parametrize("m", [3, 40])
def test_w4_scales_over_a_wide_range(m):
    """Scales from 1e-6 to 1e-2 within a row, and rows of very small and very large scales."""
    n, k, group = 130, 1024, 32
    for dtype in (BF16, E4M3):
        q, s, z = weights(n, k, group, True, BF16, 3, spread=1e-4)
        s[1] = (s[1].float() * 1e-25).to(BF16)
        s[2] = (s[2].float() * 1e25).to(BF16)
        s[3] = 0
        W, A = dense64(q, s, z, k, group)
        x, xs = rows(m, k, dtype, 4)
        y = sw().W4Matrix(q, s, z, group=group)(x, xs)
        assert (y[:, 3] == 0).all()
        for part in ([0] + list(range(4, n)), [1], [2]):
            check_product(y[:, part], x, xs, W[part], A[part], BF16)


@pytest.mark.parametrize("m", [1, 8, 33, 200])
def test_w4_special_values_stay_in_their_row(m):
    n, k = 150, 500
    q, s, z = weights(n, k, 128, False, BF16, 3)
    W, A = dense64(q, s, z, k, 128)
    matrix = sw().W4Matrix(q, s, None, k=k)
    x, _ = rows(m + 2, k, BF16, 4)
    x[0, 3], x[m + 1, k - 1] = float("nan"), float("inf")
    y = matrix(x)
    assert torch.isnan(y[0]).all() and not torch.isfinite(y[m + 1]).any()
    w = U[BF16] if m + 2 > 16 else 0.0
    want, size = x[1:m + 1].double() @ W.t(), x[1:m + 1].double().abs() @ A.t()
    assert ((y[1:m + 1].double() - want).abs() <= U[BF16] * want.abs() + (k * 2.0 ** -23 + w) * size).all()
    # rows of zeros give zeros
    assert (matrix(torch.zeros(m, k, device="cuda", dtype=BF16)) == 0).all()


@pytest.mark.parametrize("m", [1, 7, 64, 300])
def test_w4_gives_the_same_bits_every_time_and_for_a_row_alone_in_its_launch_shape(m):
    q, s, z = weights(900, 2100, 64, True, BF16, 8)
    matrix = sw().W4Matrix(q, s, z, k=2100, group=64)
    x, _ = rows(m, 2100, BF16, 1)
    y = matrix(x)
    for _ in range(5):
        assert torch.equal(matrix(x), y)


def test_w4_offsets_past_32_bits():
    """Rows of x and of the result more than 2^31 elements apart."""
    n, k, far = 192, 256, 2 ** 31 + 64
    q, s, z = weights(n, k, 128, False, BF16, 2)
    W, A = dense64(q, s, z, k, 128)
    matrix = sw().W4Matrix(q, s, z, k=k)
    xbuf = torch.zeros(2 * far + 512, dtype=torch.uint8, device="cuda").view(E4M3)
    obuf = torch.zeros(far + 512, dtype=BF16, device="cuda")
    x, xs = rows(2, k, E4M3, 3)
    xv = xbuf.as_strided((2, k), (far, 1))
    xv.view(torch.uint8).copy_(x.view(torch.uint8))
    out = obuf.as_strided((2, n), (far, 1))
    matrix(xv, xs, out=out)
    check_product(out.contiguous(), x, xs, W, A, BF16)
    # ... and of the row operators
    q8, s8 = sw().rms_norm_quant(out, torch.ones(n, device="cuda", dtype=BF16), EPS)
    check_rows(q8, s8, norm64(out.contiguous(), torch.ones(n, device="cuda")))


def test_w4_no_rows():
    q, s, z = weights(10, 64, 32, False, F16, 2)
    assert sw().W4Matrix(q, s, group=32)(torch.empty(0, 64, device="cuda", dtype=F16)).shape == (0, 10)


# ---- together ------------------------------------------------------------------------------------------------------

def block(width, inner, group, seed):
    from paper_1202_3173_b200.feed_forward import FeedForward, W4Matrix
    made, dense = [], []
    for n, k in ((2 * inner, width), (width, inner)):
        q, s, z = weights(n, k, group, True, BF16, seed + n)
        made.append(W4Matrix(q, s, z, k=k, group=group))
        dense.append(dense64(q, s, z, k, group)[0])
    norm = (1 + 0.1 * torch.randn(width, device="cuda", generator=gen(seed))).to(BF16)
    return FeedForward(norm, *made), norm, dense


@pytest.mark.parametrize("m", [1, 5, 40])
@pytest.mark.parametrize("width,inner,group", [(256, 512, 128), (133, 301, 32)])
def test_feed_forward_block(m, width, inner, group):
    ff, norm, (w1, w2) = block(width, inner, group, 3)
    g = gen(m)
    x, r = (torch.randn(m, width, device="cuda", generator=g).to(BF16) for _ in range(2))
    y, h = ff(x, r)
    assert torch.equal(h, (x.float() + r.float()).to(BF16))
    n = norm64(x, norm, r)
    a, b = (n @ w1.t()).split(inner, 1)
    want = (a * torch.special.expit(a) * b) @ w2.t()
    # two roundings to e4m3 of relative size 2^-4 / sqrt(3) at most each (root mean square), the first entering both factors of the gate
    assert (y.double() - want).norm() <= 2.0 ** -4 * 3 * want.norm()


def test_feed_forward_on_another_stream_and_in_a_graph():
    ff, _, _ = block(256, 512, 128, 3)
    x, r = (torch.randn(4, 256, device="cuda", generator=gen(1)).to(BF16) for _ in range(2))
    want, _ = ff(x, r)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            got, _ = ff(x, r)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held, _ = ff(x, r)
    other = torch.randn(4, 256, device="cuda", generator=gen(2)).to(BF16)
    eager, _ = ff(other, r)
    x.copy_(other)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, eager)


def test_operators_keep_stream_order():
    """Inputs rewritten and outputs consumed between calls of one stream, nothing waited for."""
    ff, _, _ = block(512, 1024, 128, 3)
    xs = [torch.randn(4, 512, device="cuda", generator=gen(i)).to(BF16) for i in range(6)]
    r = torch.zeros_like(xs[0])
    want = [ff(x, r)[0].clone() for x in xs]
    torch.cuda.synchronize()
    held, got = torch.empty_like(xs[0]), []
    for _ in range(10):
        for i, x in enumerate(xs):
            held.copy_(x)
            y, _ = ff(held, r)
            got.append((i, y))
    torch.cuda.synchronize()
    for i, y in got:
        assert torch.equal(y, want[i])


# ---- refusals -------------------------------------------------------------------------------------------------------

def test_refusals_of_shapes_types_and_devices():
    m = sw()
    x = torch.randn(4, 64, device="cuda").to(BF16)
    w = torch.ones(64, device="cuda", dtype=BF16)
    q, s = m.quant_rows(4, 64)
    bad = [lambda: m.rms_norm_quant(x.cpu(), w), lambda: m.rms_norm_quant(x, w.cpu()), lambda: m.rms_norm_quant(x, w[:63]),
           lambda: m.rms_norm_quant(x, w.float()), lambda: m.rms_norm_quant(x.double(), w.double()), lambda: m.rms_norm_quant(x[0], w),
           lambda: m.rms_norm_quant(x.t(), w[:4]), lambda: m.rms_norm_quant(x, w, residual=x[:3]), lambda: m.rms_norm_quant(x, w, residual=x.half()),
           lambda: m.rms_norm_quant(x, w, out=(q, s[:3])), lambda: m.rms_norm_quant(x, w, out=(q[:, :63], s)), lambda: m.rms_norm_quant(x, w, out=(q, s, x)),
           lambda: m.silu_mul_quant(x, x[:, :63]), lambda: m.silu_mul_quant(x, x.float()), lambda: m.silu_mul_quant(x, x, out=(q.float(), s))]
    qq, ss, zz = weights(32, 64, 32, True, BF16, 1)
    W = m.W4Matrix(qq, ss, zz, group=32)
    bad += [lambda: m.W4Matrix(qq.int(), ss, zz, group=32), lambda: m.W4Matrix(qq.cpu(), ss, zz, group=32), lambda: m.W4Matrix(qq, ss.float(), zz, group=32),
            lambda: m.W4Matrix(qq, ss[:, :1], zz, group=32), lambda: m.W4Matrix(qq, ss, zz[:31], group=32), lambda: m.W4Matrix(qq, ss, zz, k=70, group=32),
            lambda: W(x[:, :63]), lambda: W(x.float()), lambda: W(x.cpu()), lambda: W(x, s[:3]), lambda: W(x, s.double()),
            lambda: W(x, out=torch.empty(4, 31, device="cuda", dtype=BF16)), lambda: W(x, out=torch.empty(4, 32, device="cuda")),
            lambda: W(x, out=torch.empty(4, 32, device="cuda", dtype=BF16), dtype=F16), lambda: m.FeedForward(w, W, W)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("refusal %d" % i)
    W.close()
    with pytest.raises(ValueError):
        W(x)


def test_refusals_at_the_c_boundary():
    x = torch.randn(4, 64, device="cuda").to(BF16)
    w = torch.ones(64, device="cuda", dtype=BF16)
    q, s = sw().quant_rows(4, 64)
    p = lambda t: t.data_ptr()  # noqa: E731
    b = binding
    norm = lambda **k: b.strassen_rms_norm_quant(**{**dict(m=4, k=64, type=0, x=p(x), ldx=64, residual=0, ldr=0, weight=p(w), eps=1e-6, sum=0, lds=0,  # noqa: E731
                                                           q=p(q), ldq=64, scale=p(s)), **k})
    for status, change in ((-1, dict(m=-1)), (-1, dict(k=0)), (-1, dict(type=3)), (-1, dict(type=9)), (-1, dict(x=0)), (-1, dict(weight=0)), (-1, dict(q=0)),
                           (-1, dict(scale=0)), (-1, dict(ldx=63)), (-1, dict(ldq=63)), (-1, dict(eps=-1.0)), (-1, dict(eps=float("nan"))),
                           (-1, dict(residual=p(x), ldr=64)), (-1, dict(sum=p(x), lds=64)), (-5, dict(x=p(x) + 1)), (-5, dict(scale=p(s) + 2)), (-5, dict(weight=p(w) + 1)),
                           (-4, dict(q=p(x))), (-4, dict(scale=p(x))), (-4, dict(q=p(w))), (-4, dict(residual=p(x), ldr=64, sum=p(x) + 128, lds=64))):
        with pytest.raises(StrassenError) as e:
            norm(**change)
        assert e.value.status == status, (change, str(e.value))
    norm(m=0, x=0, q=0)
    qq, ss, zz = weights(32, 64, 32, True, BF16, 1)
    h = b.strassen_w4_create(32, 64, 32, 0, True)
    out = torch.empty(4, 32, device="cuda", dtype=BF16)
    mem = torch.empty(b.strassen_w4_bytes(h), dtype=torch.uint8, device="cuda")
    mul = lambda **k: b.strassen_w4_matmul(**{**dict(matrix=h, m=4, type=0, x=p(x), ldx=64, x_scale=0, out_type=0, out=p(out), ldo=32), **k})  # noqa: E731
    with pytest.raises(StrassenError):
        mul()                                            # not laid out yet
    pack = lambda **k: b.strassen_w4_pack(**{**dict(matrix=h, q=p(qq), ldq=32, scales=p(ss), lds=2, zeros=p(zz), ldz=2, packed=p(mem)), **k})  # noqa: E731
    for status, change in ((-1, dict(q=0)), (-1, dict(scales=0)), (-1, dict(zeros=0)), (-1, dict(packed=0)), (-1, dict(ldq=31)), (-1, dict(lds=1)), (-1, dict(ldz=1)),
                           (-5, dict(packed=p(mem) + 16)), (-5, dict(scales=p(ss) + 1)), (-1, dict(matrix=0))):
        with pytest.raises(StrassenError) as e:
            pack(**change)
        assert e.value.status == status, (change, str(e.value))
    pack()
    for status, change in ((-1, dict(matrix=0)), (-1, dict(m=-1)), (-1, dict(type=2)), (-1, dict(out_type=2)), (-1, dict(out_type=3)), (-1, dict(x=0)), (-1, dict(out=0)),
                           (-1, dict(ldx=63)), (-1, dict(ldo=31)), (-5, dict(x=p(x) + 1)), (-5, dict(out=p(out) + 1)), (-5, dict(x_scale=p(s) + 1)),
                           (-4, dict(out=p(x))), (-4, dict(out=p(mem)))):
        with pytest.raises(StrassenError) as e:
            mul(**change)
        assert e.value.status == status, (change, str(e.value))
    mul()
    mul(m=0, x=0)
    torch.cuda.synchronize()
    b.strassen_w4_destroy(h)


def test_device_status_is_clean():
    q, s, z = weights(256, 1024, 128, False, BF16, 2)
    sw().W4Matrix(q, s)(rows(64, 1024, BF16, 1)[0])
    binding.strassen_device_status()


@pytest.mark.parametrize("m,n,k", [(20, 4096, 8192), (60, 4096, 8192), (112, 4096, 16384), (130, 512, 20000), (200, 4096, 16384), (900, 4096, 3000), (300, 2100, 256)])
def test_w4_many_launches(m, n, k):
    """Every number of rows has rings of its own depths: the same result from each of many launches, and no wait that ran out."""
    q, s, z = weights(n, k, 64, True, BF16, 3)
    matrix = sw().W4Matrix(q, s, z, group=64)
    x, _ = rows(m, k, BF16, 4)
    want, out = matrix(x), torch.empty(m, n, device="cuda", dtype=BF16)
    bad = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(300):
        matrix(x, out=out)
        bad += (out != want).sum()
    assert int(bad) == 0
    binding.strassen_device_status()


# ---- routing ---------------------------------------------------------------------------------------------------------

def route64(logits, top, score, bias, groups, top_groups, renormalize, factor):
    """(ids, weights, margin): the definition in 64 bits; margin: by how much the closest choice of each token was made."""
    l = logits.double().cpu()
    tokens, e = l.shape
    left_out = ~(l > -float("inf"))
    if score == "softmax":
        s = torch.softmax(l.masked_fill(left_out, -float("inf")), 1).nan_to_num(0.0)
        key = s + bias.double().cpu() if bias is not None else l
    else:
        s = torch.special.expit(l)
        key = s + bias.double().cpu() if bias is not None else s
    ids, weights, margin = torch.full((tokens, top), -1), torch.zeros(tokens, top, dtype=torch.float64), torch.full((tokens,), float("inf"), dtype=torch.float64)
    size = e // groups
    for t in range(tokens):
        keys = {i: float(key[t, i]) for i in range(e) if not left_out[t, i] and float(key[t, i]) > -float("inf")}

        def pick(rated, n):
            order = sorted(rated, key=lambda i: (-rated[i], i))
            for a, b in zip(order[:n], order[1:n + 1]):
                if rated[a] != rated[b]:
                    margin[t] = min(margin[t], rated[a] - rated[b])
            return order[:n]
        if groups > 1:
            rated = {}
            for g in range(groups):
                k = sorted((v for i, v in keys.items() if i // size == g), reverse=True)
                if k:
                    rated[g] = k[0] if score == "softmax" or len(k) == 1 else k[0] + k[1]
            kept = pick(rated, top_groups)
            keys = {i: v for i, v in keys.items() if i // size in kept}
        chosen = pick(keys, top)
        for j, i in enumerate(chosen):
            ids[t, j], weights[t, j] = i, s[t, i]
    if renormalize:
        total = weights.sum(1, keepdim=True)
        weights = torch.where(total > 0, weights / total, torch.zeros_like(weights))
    return ids, weights * factor, margin


def check_route(logits, top, score="softmax", bias=None, groups=1, top_groups=1, renormalize=True, factor=1.0):
    ids, weights = sw().route_experts(logits, top, score=score, bias=bias, groups=groups, top_groups=top_groups, renormalize=renormalize, factor=factor)
    want, w64, margin = route64(logits, top, score, bias, groups, top_groups, renormalize, factor)
    clear = margin > 2e-6                        # scores in 32 bits: errors of a few 2^-24, of a sum of two twice that
    assert clear.any()
    assert torch.equal(ids.cpu()[clear].long(), want[clear])
    assert ((weights.double().cpu()[clear] - w64[clear]).abs() <= 1e-5 * w64[clear] + 1e-12).all()
    # every token's ids are distinct and in range, clear or not
    for row in ids.cpu()[~clear].tolist():
        got = [i for i in row if i >= 0]
        assert len(set(got)) == len(got) and all(i < logits.shape[1] for i in got)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("tokens,experts,top", [(1, 1, 1), (1, 8, 2), (5, 31, 4), (9, 32, 32), (7, 33, 5), (64, 64, 8), (3, 100, 6), (130, 128, 8), (2, 256, 8), (17, 257, 16), (5, 512, 10), (4, 1000, 32), (2, 1024, 8)])
def test_route(tokens, experts, top, dtype):
    g = gen(experts + tokens)
    logits = (torch.randn(tokens, experts, device="cuda", generator=g) * 2).to(dtype)
    bias = 0.1 * torch.randn(experts, device="cuda", generator=g)
    for score in ("softmax", "sigmoid"):
        for b in (None, bias):
            check_route(logits, top, score, b, renormalize=b is None, factor=2.5 if b is None else 1.0)


@pytest.mark.parametrize("experts,groups,top_groups,top", [(8, 8, 3, 3), (32, 32, 5, 5), (64, 8, 4, 8), (256, 8, 4, 8), (96, 3, 2, 6), (160, 16, 1, 10), (1024, 32, 7, 32), (60, 2, 2, 7), (512, 4, 3, 16)])
def test_route_groups(experts, groups, top_groups, top):
    g = gen(experts + groups)
    logits = torch.randn(40, experts, device="cuda", generator=g)
    bias = 0.2 * torch.randn(experts, device="cuda", generator=g)
    for score in ("softmax", "sigmoid"):
        for b in (None, bias):
            check_route(logits, top, score, b, groups, top_groups)


def test_route_ties_go_to_the_lowest_index():
    logits = torch.zeros(3, 70, device="cuda")
    logits[1, 40:] = 1.0
    logits[2, ::7] = -0.0
    ids, weights = sw().route_experts(logits, 4)
    assert ids.tolist() == [[0, 1, 2, 3], [40, 41, 42, 43], [0, 1, 2, 3]]
    assert torch.allclose(weights, torch.full_like(weights, 0.25))
    ids, _ = sw().route_experts(torch.zeros(2, 64, device="cuda"), 3, score="sigmoid", groups=8, top_groups=2)
    assert ids.tolist() == [[0, 1, 2]] * 2


def test_route_experts_left_out():
    inf = float("inf")
    logits = torch.randn(6, 40, device="cuda", generator=gen(1))
    logits[0, 3:] = -inf                          # three left for five
    logits[1] = -inf                              # none
    logits[2, 5], logits[2, 6] = float("nan"), -inf
    logits[3, 7] = inf
    for score in ("softmax", "sigmoid"):
        for groups in (1, 4):
            check_route(logits[[0, 1, 2, 4, 5]], 5, score, groups=groups, top_groups=min(groups, 2))
            ids, weights = sw().route_experts(logits, 5, score=score, groups=groups, top_groups=min(groups, 2))
            assert (ids[1] == -1).all() and (weights[1] == 0).all() and ids[3, 0] == 7
            assert (ids[0] >= 0).sum() == 3 and torch.isfinite(weights).all()
    ids, weights = sw().route_experts(torch.full((1, 16), -200.0, device="cuda"), 4, score="sigmoid")      # scores that are all 0
    assert ids.tolist() == [[0, 1, 2, 3]] and (weights == 0).all()


def test_route_strides_and_no_tokens():
    wide = torch.randn(9, 77, device="cuda", generator=gen(3)).to(BF16)
    check_route(wide[:, 3:69], 6)
    ids, weights = sw().route_experts(wide[:0, :64], 6)
    assert ids.shape == (0, 6) and weights.shape == (0, 6)


# ---- products of experts ---------------------------------------------------------------------------------------------

def experts_case(experts, n, k, group, zeros, sdtype, seed):
    q, s, z = weights(experts * n, k, group, zeros, sdtype, seed)
    W, A = dense64(q, s, z, k, group)
    shape = lambda t: t.view(experts, n, -1)  # noqa: E731
    matrices = sw().W4Experts(shape(q), shape(s), shape(z) if z is not None else None, k=k, group=group)
    return matrices, W.view(experts, n, k), A.view(experts, n, k)


def check_experts(matrices, W, A, x, xs, ids, factor, out_dtype, y):
    """y against the sums, with the tolerances of the products; a sum of ids adds the rounding of its own."""
    tokens, top = ids.shape
    experts, n, k = W.shape
    xd = x.double() if xs is None else x.double() * xs.double()[:, None]
    if x.shape[0] == tokens and top > 1 or x.shape[0] == tokens:
        xd = xd.repeat_interleave(top, 0) if x.shape[0] != tokens * top else xd
    want = torch.zeros(tokens * top, n, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(want)
    flat = ids.flatten().long()
    for e in range(experts):
        at = (flat == e).nonzero()[:, 0]
        want[at], size[at] = xd[at] @ W[e].t(), xd[at].abs() @ A[e].t()
    if factor is not None:
        f = factor.double()[..., None]
        want, size = (want.view(tokens, top, n) * f).sum(1), (size.view(tokens, top, n) * f.abs()).sum(1)
    w = 0.0 if tokens * top <= 32 else U[BF16] if x.dtype == BF16 else U[F16]
    assert y.dtype == out_dtype and y.shape == want.shape and torch.isfinite(y).all()
    err = (y.double() - want).abs()
    lim = U[out_dtype] * want.abs() + ((k + top) * 2.0 ** -23 + w) * size + (6e-8 if out_dtype == F16 else 0)
    assert (err <= lim).all(), float((err - lim).max())
    assert err.norm() <= (2 * U[out_dtype] + 2 * w + k * 2.0 ** -23) * want.norm() + 6e-8 * err.numel() ** 0.5


EXPERT_SHAPES = [(1, 1, 4, 16, 64), (1, 8, 16, 200, 300), (4, 2, 3, 129, 257), (3, 8, 64, 128, 512), (2, 16, 40, 100, 1000), (5, 8, 10, 130, 200), (33, 1, 7, 64, 96),
                 (40, 4, 6, 300, 140), (200, 2, 3, 257, 400), (700, 3, 20, 130, 256), (300, 8, 300, 40, 64), (64, 32, 40, 96, 128)]


@pytest.mark.parametrize("group,zeros", [(32, True), (64, False), (128, True)])
@pytest.mark.parametrize("tokens,top,experts,n,k", EXPERT_SHAPES)
def test_experts(tokens, top, experts, n, k, group, zeros):
    g = gen(tokens + k)
    ids = torch.rand(tokens, experts, device="cuda", generator=g).pow(3).argsort(1)[:, :top].to(torch.int32).contiguous() if top <= experts else \
        torch.randint(0, experts, (tokens, top), device="cuda", generator=g, dtype=torch.int32)
    factor = torch.rand(tokens, top, device="cuda", generator=g)
    for dtype, out_dtype, sdtype in ((BF16, BF16, BF16), (F16, F16, F16), (E4M3, BF16, BF16)):
        matrices, W, A = experts_case(experts, n, k, group, zeros, sdtype, n + k)
        for m in (tokens, tokens * top):
            x, xs = rows(m, k, dtype, m)
            for f in (None, factor):
                check_experts(matrices, W, A, x, xs, ids, f, out_dtype, matrices(x, ids, xs, weights=f, dtype=out_dtype))


@pytest.mark.parametrize("tokens", [3, 50])
def test_experts_ids_that_name_none(tokens):
    n, k, experts, top = 150, 300, 5, 4
    matrices, W, A = experts_case(experts, n, k, 64, True, BF16, 3)
    g = gen(tokens)
    ids = torch.randint(-2, experts + 2, (tokens, top), device="cuda", generator=g, dtype=torch.int32)
    ids[1] = -1                                  # a token without any
    ids[2, 0] = 2 ** 31 - 1
    factor = torch.rand(tokens, top, device="cuda", generator=g)
    x, _ = rows(tokens, k, BF16, 5)
    for f in (None, factor):
        y = matrices(x, ids, weights=f)
        check_experts(matrices, W, A, x, None, ids, f, BF16, y)
        assert (y.view(tokens, -1)[1] == 0).all()
    y = matrices(x, torch.full_like(ids, -1))
    assert (y == 0).all()


@pytest.mark.parametrize("tokens", [2, 60])
def test_experts_strides(tokens):
    n, k, experts, top = 140, 333, 6, 3
    q, s, z = weights(experts * n, k, 64, True, BF16, 9)
    W, A = dense64(q, s, z, k, 64)
    qs, ss, zs = (strided(t, 5, 1, 0).unflatten(0, (experts, n)) for t in (q, s, z))
    matrices = sw().W4Experts(qs, ss, zs, k=k, group=64)
    ids = torch.randint(0, experts, (tokens, top), device="cuda", generator=gen(2), dtype=torch.int32)
    for dtype in (BF16, E4M3):
        x, xs = rows(tokens * top, k, dtype, 3)
        out = strided(torch.zeros(tokens * top, n, device="cuda").to(BF16), 3, 1, 7.0)
        matrices(strided(x, 3, 1), ids, xs, out=out)
        check_experts(matrices, W.view(experts, n, k), A.view(experts, n, k), x, xs, ids, None, BF16, out)
        assert (out.as_strided((tokens * top - 1, 3), (n + 3, 1), out.storage_offset() + n) == 7).all()


def test_experts_many_launches_and_special_rows():
    """The same bits each time; a NaN in one row of x stays in that row's results, although other rows share its tile."""
    experts, top, tokens = 8, 2, 300
    matrices, W, A = experts_case(experts, 512, 1024, 128, False, BF16, 3)
    g = gen(1)
    ids = torch.rand(tokens, experts, device="cuda", generator=g).argsort(1)[:, :top].to(torch.int32).contiguous()
    factor = torch.rand(tokens, top, device="cuda", generator=g)
    x, _ = rows(tokens, 1024, BF16, 3)
    x[17, 5] = float("nan")
    fine = torch.arange(tokens, device="cuda") != 17
    want = matrices(x, ids, weights=factor)
    assert torch.isnan(want[17]).all() and torch.isfinite(want[fine]).all()
    for _ in range(100):
        assert torch.equal(matrices(x, ids, weights=factor)[fine], want[fine])
    binding.strassen_device_status()


def test_experts_block():
    from paper_1202_3173_b200.feed_forward import ExpertsFeedForward
    width, inner, experts, top = 128, 192, 6, 2
    up, W1, _ = experts_case(experts, 2 * inner, width, 64, True, BF16, 3)
    down, W2, _ = experts_case(experts, width, inner, 64, True, BF16, 4)
    g = gen(3)
    norm = (1 + 0.1 * torch.randn(width, device="cuda", generator=g)).to(BF16)
    router = torch.randn(experts, width, device="cuda", generator=g).to(BF16)
    block_ = ExpertsFeedForward(norm, router, up, down, top, score="sigmoid")
    for tokens in (1, 70):
        x, r = (torch.randn(tokens, width, device="cuda", generator=g).to(BF16) for _ in range(2))
        y, h = block_(x, r)
        q, s, _ = sw().rms_norm_quant(x, norm, EPS, residual=r)
        v = q.double() * s.double()[:, None]
        ids, f = sw().route_experts((v @ router.double().t()).float(), top, score="sigmoid")
        want = torch.zeros(tokens, width, dtype=torch.float64, device="cuda")
        for t in range(tokens):
            for j in range(top):
                e = int(ids[t, j])
                a, b = (W1[e] @ v[t]).split(inner)
                want[t] += float(f[t, j]) * (W2[e] @ (a * torch.special.expit(a) * b))
        # the inner rows are rounded to bf16 and then to e4m3
        assert (y.double() - want).norm() <= 2.0 ** -4 * want.norm()


def test_refusals_of_routing_and_experts():
    m = sw()
    l = torch.randn(4, 64, device="cuda")
    ids, f = m.route_experts(l, 4)
    q, s, z = weights(6 * 32, 64, 32, True, BF16, 1)
    E = m.W4Experts(q.view(6, 32, -1), s.view(6, 32, -1), z.view(6, 32, -1), group=32)
    x = torch.randn(4, 64, device="cuda").to(BF16)
    bad = [lambda: m.route_experts(l.cpu(), 4), lambda: m.route_experts(l.double(), 4), lambda: m.route_experts(l[0], 4), lambda: m.route_experts(l, 4, score="tanh"),
           lambda: m.route_experts(l, 4, bias=l[0, :63]), lambda: m.route_experts(l, 4, bias=l[0].half()), lambda: m.route_experts(l, 4, out=(ids.long(), f)),
           lambda: m.route_experts(l, 4, out=(ids, f[:, :3])), lambda: m.route_experts(l.t(), 4),
           lambda: E(x, ids.long()), lambda: E(x, ids[0]), lambda: E(x[:3], ids), lambda: E(x[:, :63], ids), lambda: E(x, ids, weights=f[:, :3]), lambda: E(x, ids, weights=f.double()),
           lambda: E(x, ids, f[:, 0]), lambda: E(x, ids, out=torch.empty(4, 32, device="cuda", dtype=BF16)), lambda: E(x, ids, weights=f, out=torch.empty(16, 32, device="cuda", dtype=BF16)),
           lambda: E(x.float(), ids), lambda: E(x, ids.cpu()), lambda: m.W4Experts(q, s, z, group=32), lambda: m.W4Experts(q.view(6, 32, -1), s.view(3, 64, -1), None, group=32),
           lambda: m.W4Experts(q.view(6, 32, -1).transpose(0, 1), s.view(6, 32, -1).transpose(0, 1), None, group=32)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("refusal %d" % i)
    many, xs, ys = torch.zeros(100, 4, device="cuda", dtype=torch.int32), torch.zeros(100, 64, device="cuda", dtype=BF16), torch.zeros(400, 32, device="cuda", dtype=BF16)
    for call in (lambda: m.route_experts(l, 65), lambda: m.route_experts(l, 33), lambda: m.route_experts(l, 4, groups=7), lambda: m.route_experts(l, 9, groups=8, top_groups=1),
                 lambda: binding.strassen_w4_matmul(E.handle, 4, 0, x.data_ptr(), 64, 0, 0, l.data_ptr(), 32),
                 lambda: binding.strassen_w4_experts(E.handle, 4, 33, ids.data_ptr(), 0, x.data_ptr(), 64, False, 0, 0, 0, l.data_ptr(), 32),
                 lambda: binding.strassen_w4_experts(E.handle, 100, 4, many.data_ptr(), 0, xs.data_ptr(), 64, False, 0, 0, 0, ys.data_ptr(), 32)):
        with pytest.raises(StrassenError) as e:
            call()
        assert e.value.status in (-1, -3)
