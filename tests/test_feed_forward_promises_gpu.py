"""Feed-forward operators: refusals and promises beside the formulas (aliases, capture, gradients, types of blocks, bits of a row in a batch)."""
import pytest
import torch

from paper_1202_3173_b200 import StrassenError, binding

from .test_feed_forward_gpu import BF16, E4M3, EPS, F16, F32, check_rows, dense64, gen, norm64, rows, strided, weights

pytestmark = pytest.mark.gpu


def sw():
    import paper_1202_3173_b200 as m
    return m


def test_a_workspace_in_the_weights_or_an_argument_is_refused():
    """More than 16 rows in e4m3, which need a workspace: in the laid-out weights it would overwrite them for this and every later call."""
    m, n, k = 20, 1024, 512
    q, s, z = weights(n, k, 128, False, BF16, 1)
    matrix = sw().W4Matrix(q, s)
    x, xs = rows(m, k, E4M3, 2)
    out = torch.empty(m, n, device="cuda", dtype=BF16)
    need = binding.strassen_w4_workspace_bytes(matrix.handle, m, binding.STRASSEN_E4M3, x.data_ptr(), k)
    assert 0 < need < matrix.nbytes
    before = matrix._packed.clone()
    for at in (matrix._packed, x, xs, out):
        with pytest.raises(StrassenError) as e:
            binding.strassen_w4_matmul(matrix.handle, m, binding.STRASSEN_E4M3, x.data_ptr(), k, xs.data_ptr(), binding.STRASSEN_BF16, out.data_ptr(), n, at.data_ptr(),
                                       need, torch.cuda.current_stream().cuda_stream)
        assert e.value.status == -4, str(e.value)
    torch.cuda.synchronize()
    assert torch.equal(matrix._packed, before)


def test_a_matrix_collected_during_a_capture_leaves_it_whole():
    q, s, z = weights(300, 512, 64, True, BF16, 3)
    x, _ = rows(4, 512, BF16, 4)
    kept, dropped = (sw().W4Matrix(q, s, z, group=64) for _ in range(2))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        want = dropped(x)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        del dropped
        got = kept(x)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_the_memory_of_a_matrix_is_not_reused_under_products_on_other_streams():
    n, k = 1024, 4096
    q, s, z = weights(n, k, 128, False, BF16, 5)
    x, _ = rows(4, k, BF16, 6)
    want = sw().W4Matrix(q, s)(x)
    torch.cuda.synchronize()
    matrix = sw().W4Matrix(q, s)
    nbytes, side = matrix.nbytes, torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100000000)             # some 50 ms
        got = matrix(x)
    del matrix
    others = [torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    del others


def test_gradients_are_refused_and_not_dropped():
    x = torch.randn(4, 64, device="cuda")
    w, leaf = torch.ones(64, device="cuda"), torch.randn(4, 64, device="cuda", requires_grad=True)
    q, s, _ = weights(32, 64, 32, False, BF16, 1)
    m = sw()
    matrix, experts = m.W4Matrix(q, s, group=32), m.W4Experts(q.view(2, 16, -1), s.view(2, 16, -1), group=32)
    ids, factor = m.route_experts(x[:, :2], 1)
    half, leaf16, scale = x.to(BF16), leaf.detach().to(BF16).requires_grad_(), torch.ones(4, device="cuda", requires_grad=True)
    calls = [lambda: m.rms_norm_quant(leaf, w), lambda: m.rms_norm_quant(x, w.clone().requires_grad_()), lambda: m.rms_norm_quant(x, w, residual=leaf),
             lambda: m.rms_norm_quant(x, w, residual=x, out=m.quant_rows(4, 64) + (leaf,)), lambda: m.silu_mul_quant(x, leaf), lambda: m.silu_mul_quant(leaf, x),
             lambda: m.route_experts(leaf, 2), lambda: m.route_experts(x, 2, bias=torch.zeros(64, device="cuda", requires_grad=True)),
             lambda: matrix(leaf16), lambda: matrix(half, scale), lambda: experts(leaf16, ids), lambda: experts(half, ids, scale),
             lambda: experts(half, ids, weights=factor.clone().requires_grad_())]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="requires grad"):
            call()
            pytest.fail("call %d" % i)
        with torch.no_grad():
            call()
        with torch.inference_mode():
            call()


def test_tensors_that_are_written_count_as_modified():
    x, r, w = torch.randn(4, 64, device="cuda"), torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda", requires_grad=True)
    m = sw()
    loss = (r * w).sum()                         # saves r
    m.rms_norm_quant(x, torch.ones(64, device="cuda"), residual=r, out=m.quant_rows(4, 64) + (r,))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    q, s, _ = weights(32, 64, 32, False, BF16, 1)
    matrix, experts = m.W4Matrix(q, s, group=32), m.W4Experts(q.view(2, 16, -1), s.view(2, 16, -1), group=32)
    ids, factor = m.route_experts(x[:, :2], 1)
    eight, out, each = m.quant_rows(4, 64), torch.empty(4, 32, device="cuda", dtype=BF16), torch.empty(4, 16, device="cuda", dtype=BF16)
    written = [*eight, out, each, ids, factor]
    before = [t._version for t in written]
    m.silu_mul_quant(x, r, out=eight)
    m.route_experts(x[:, :2], 1, out=(ids, factor))
    matrix(x.to(BF16), out=out)
    experts(x.to(BF16), ids, out=each)
    assert all(t._version > v for t, v in zip(written, before))


@pytest.mark.parametrize("m", [1, 40])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_blocks_of_every_type_follow_one_another(m, dtype):
    """A block's output goes into the next block beside its residual stream."""
    width, inner, experts = 192, 256, 4
    g = gen(m)
    made = []
    for n, k in ((2 * inner, width), (width, inner)):
        q, s, _ = weights(experts * n, k, 64, False, BF16, n)
        made.append((sw().W4Matrix(q[:n], s[:n], group=64), sw().W4Experts(q.view(experts, n, -1), s.view(experts, n, -1), group=64)))
    norm = torch.ones(width, device="cuda", dtype=dtype)
    router = torch.randn(experts, width, device="cuda", generator=g).to(dtype)
    blocks = [sw().FeedForward(norm, made[0][0], made[1][0]), sw().ExpertsFeedForward(norm, router, made[0][1], made[1][1], 2), sw().FeedForward(norm, made[0][0], made[1][0])]
    y, h = (torch.randn(m, width, device="cuda", generator=g).to(dtype) for _ in range(2))
    for block in blocks:
        total = y.float() + h.float()
        y, h = block(y, h)
        assert y.dtype == dtype and h.dtype == dtype and torch.isfinite(y).all()
        assert torch.equal(h, total.to(dtype))


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("k", [1, 9, 70, 140, 255])
def test_laid_out_positions_past_the_inner_size_are_worth_nothing(k, group):
    """The laid-out tiles as their description has them: 128 x 128 nibbles in 16-byte chunks, then scales and zero points of each group."""
    n = 130
    q, s, z = weights(n, k, group, True, BF16, k)
    z[:] = z % 8                                 # no zero point is 8
    matrix = sw().W4Matrix(q, s, z, k=k, group=group)
    per_tile, deep = 128 // group, -(-k // 128)
    size = 8192 + per_tile * 128 * 3
    data, hq, hz = matrix._packed.cpu(), q.cpu(), z.cpu()
    for tile in range(2 * deep):
        t = data[tile * size:(tile + 1) * size]
        scale = t[8192:8192 + per_tile * 256].view(torch.int16)
        zero = t[8192 + per_tile * 256:]
        for r in range(0, 128, 5):
            place = (r & ~15) | ((r & 7) << 1) | (r >> 3 & 1)
            for c in range(4):
                at = (r >> 3) * 512 + (r & 7) * 64 + (c ^ (r >> 1 & 3)) * 16
                for w in range(4):
                    word = int(t[at + 4 * w:at + 4 * w + 4].view(torch.int32)) & 0xffffffff
                    for i in range(8):
                        inner = 32 * w + 8 * c + i
                        row, col, g = tile // deep * 128 + r, tile % deep * 128 + inner, inner // group * 128 + place
                        nibble = word >> (4 * (i >> 1) + 16 * (i & 1)) & 15
                        if row < n and col < k:
                            assert nibble == int(hq[row, col // 2]) >> 4 * (col & 1) & 15 and int(zero[g]) == int(hz[row, col // group])
                        else:
                            assert nibble == int(zero[g]) or int(scale[g]) == 0


@pytest.mark.parametrize("n,k", [(64, 200), (4096, 16384), (900, 12345), (40, 40000)])
def test_a_row_has_the_same_bits_alone_and_among_up_to_16(n, k):
    q, s, z = weights(n, k, 64, True, BF16, 8)
    matrix = sw().W4Matrix(q, s, z, k=k, group=64)
    for dtype in (BF16, E4M3):
        x, xs = rows(16, k, dtype, 1)
        part = lambda a, b: matrix(x[a:b], None if xs is None else xs[a:b])  # noqa: E731
        want = torch.cat([part(i, i + 1) for i in range(16)])
        for m in (2, 5, 8, 9, 16):
            assert torch.equal(torch.cat([part(i, min(16, i + m)) for i in range(0, 16, m)]), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,k", [(3, 300), (3, 20000), (700, 100), (5000, 8192)])
def test_norm_whose_squares_pass_32_bits_is_nan_and_not_zeros(m, k, dtype):
    x = torch.randn(m, k, device="cuda", generator=gen(k)).to(dtype)
    x[1] *= 1e25
    w, fine = torch.ones(k, device="cuda", dtype=dtype), torch.arange(m, device="cuda") != 1
    for r in (None, torch.zeros_like(x)):
        q, s = sw().rms_norm_quant(x, w, EPS, residual=r)[:2]
        assert torch.isnan(s[1]) and torch.isnan(q[1].float()).all()
        check_rows(q[fine], s[fine], norm64(x[fine], w))


def test_experts_that_are_missing_weigh_nothing_whatever_the_factor():
    logits = torch.randn(2, 16, device="cuda", generator=gen(1))
    logits[:, 3:] = -float("inf")
    for score in ("softmax", "sigmoid"):
        ids, w = sw().route_experts(logits, 5, score=score, factor=float("inf"))
        assert (ids[:, 3:] == -1).all() and (w[:, 3:] == 0).all() and torch.isinf(w[:, :3]).all()


def test_experts_of_one_row_may_lie_at_any_distance():
    q, s, z = weights(12, 64, 32, True, BF16, 1)
    shape = lambda t: t.view(4, 3, -1)  # noqa: E731
    wide = sw().W4Experts(*(shape(t) for t in (q, s, z)), group=32)
    one = sw().W4Experts(*(shape(t)[:, :1] for t in (q, s, z)), group=32)
    x, _ = rows(4, 64, BF16, 2)
    ids = torch.arange(4, device="cuda", dtype=torch.int32)[:, None]
    assert torch.equal(one(x, ids), wide(x, ids)[:, :1])


@pytest.mark.parametrize("tokens", [1, 70])
def test_experts_block_whose_router_sees_the_unrounded_norm(tokens):
    """The experts are those of the norm in 64 bits; the products' tolerance is that of their 8-bit rows, as for the block with a matrix."""
    width, inner, experts, top = 128, 192, 6, 2
    made, dense = [], []
    for n, k in ((2 * inner, width), (width, inner)):
        q, s, z = weights(experts * n, k, 64, True, BF16, n)
        made.append(sw().W4Experts(*(t.view(experts, n, -1) for t in (q, s, z)), group=64))
        dense.append(dense64(q, s, z, k, 64)[0].view(experts, n, k))
    g = gen(3)
    norm = (1 + 0.1 * torch.randn(width, device="cuda", generator=g)).to(BF16)
    matrix = torch.randn(experts, width, device="cuda", generator=g)

    def router(h):
        v = h.float()
        return v * (v.square().mean(-1, keepdim=True) + EPS).rsqrt() * norm.float() @ matrix.t()
    block = sw().ExpertsFeedForward(norm, router, *made, top)
    x, r = (torch.randn(tokens, width, device="cuda", generator=g).to(BF16) for _ in range(2))
    y, h = block(x, r)
    v = norm64(h, norm)
    logits = v @ matrix.double().t()
    score, ids = logits.topk(top, 1)
    assert (logits.topk(top + 1, 1).values.diff(dim=1).abs() > 1e-3).all()       # no two experts are too close to tell in 32 bits
    f, v = torch.softmax(score, 1), norm64(x, norm, r)
    want = torch.zeros(tokens, width, dtype=torch.float64, device="cuda")
    for t in range(tokens):
        for j in range(top):
            a, b = (dense[0][ids[t, j]] @ v[t]).split(inner)
            want[t] += f[t, j] * (dense[1][ids[t, j]] @ (a * torch.special.expit(a) * b))
    # the roundings of the norm's rows enter both factors of the gate, those of the inner rows come on top: each 2^-4 / sqrt(3) at most, root mean square
    assert (y.double() - want).norm() <= 3 * 2.0 ** -4 * want.norm()
    for bad in (lambda h: router(h)[:, :3], lambda h: router(h)[0]):
        with pytest.raises(ValueError):
            sw().ExpertsFeedForward(norm, bad, *made, top)(x, r)
    with pytest.raises(ValueError):
        sw().ExpertsFeedForward(norm, matrix[:3], *made, top)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("pad,shift", [(0, 0), (7, 0), (1, 3)])
@pytest.mark.parametrize("k", [1025, 2048, 4099, 8192, 12345])
def test_sums_in_place_of_x_over_many_megabytes(k, pad, shift, dtype):
    """Norms with enough to do for CTAs that stay and copy ahead, the sum written over x while later rows of x are on their way."""
    g = gen(k + pad)
    m = 90000000 // (k * dtype.itemsize)
    x = strided(torch.randn(m, k, device="cuda", generator=g).to(dtype), pad, shift)
    r = torch.randn(m, k, device="cuda", generator=g).to(dtype)
    w = (1 + 0.3 * torch.randn(k, device="cuda", generator=g)).to(dtype)
    q, s = sw().quant_rows(m, k)
    want, v = (x.float() + r.float()).to(dtype), norm64(x, w, r)
    sw().rms_norm_quant(x, w, EPS, residual=r, out=(q, s, x))
    check_rows(q, s, v)
    assert torch.equal(x, want)
    binding.strassen_device_status()


@pytest.mark.parametrize("m", [40, 300])
def test_block_of_many_rows_in_a_graph(m):
    """Split inner dimension and pairs of CTAs, with the rows' conversion, captured and replayed on other inputs."""
    width, inner = 256, 4096
    made = []
    for n, k in ((2 * inner, width), (width, inner)):
        q, s, _ = weights(n, k, 128, False, BF16, n)
        made.append(sw().W4Matrix(q, s))
    block = sw().FeedForward(torch.ones(width, device="cuda", dtype=BF16), *made)
    x, r = (torch.randn(m, width, device="cuda", generator=gen(1)).to(BF16) for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held, _ = block(x, r)
    other = torch.randn(m, width, device="cuda", generator=gen(2)).to(BF16)
    want, _ = block(other, r)
    x.copy_(other)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(held, want)
    binding.strassen_device_status()
