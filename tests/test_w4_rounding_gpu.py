"""What the products with 4-bit weights do to each weight, seen through rows of x that hold a single 1: such a row's result is one column of the matrix.

No tolerance: the sum's other terms are zeros, and a weight S (Q - Z) has at most 11 + 4 bits, so it is exact in 32 bits; what is left are the
roundings that the operators promise, none up to 16 rows (32 ids), one to the type of the weights beyond, and one to the type of the result.
"""
import pytest
import torch

from paper_1202_3173_b200 import binding

pytestmark = pytest.mark.gpu

BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
N, K, GROUP = 150, 512, 32


def sw():
    import paper_1202_3173_b200 as m
    return m


def wide_weights(zeros, dtype, seed, rows=N):
    """(q, scales, zero points, S (Q - Z)): the scales of a row from 2^-13 to 8, the largest in its first group."""
    g = torch.Generator("cuda").manual_seed(seed)
    q = torch.randint(0, 256, (rows, K // 2), device="cuda", generator=g, dtype=torch.uint8)
    power = torch.randint(-13, 2, (rows, K // GROUP), device="cuda", generator=g).double()
    s = ((1 + torch.rand(rows, K // GROUP, device="cuda", generator=g).double()) * torch.exp2(power)).to(dtype)
    s[:, 0] = 8.0 * (1 - 2.0 ** -8)
    s[::3] = -s[::3]
    z = torch.randint(0, 16, s.shape, device="cuda", generator=g, dtype=torch.uint8) if zeros else None
    nibbles = torch.stack([q & 15, q >> 4], -1).view(rows, K).double()
    z64 = z.double().repeat_interleave(GROUP, 1) if zeros else 8.0
    return q, s, z, s.double().repeat_interleave(GROUP, 1) * (nibbles - z64)


def columns(product, dtype, m):
    """The matrix (N x K) from products of m rows of the unit matrix at a time."""
    x = torch.eye(K, device="cuda").to(dtype)
    return torch.cat([product(x[i:i + m]) for i in range(0, K, m)]).t()


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("scales", [BF16, F16])
@pytest.mark.parametrize("dtype", [BF16, F16, E4M3])
def test_up_to_16_rows_no_weight_is_rounded(dtype, scales, zeros):
    q, s, z, w = wide_weights(zeros, scales, 1)
    matrix = sw().W4Matrix(q, s, z, group=GROUP)
    for m in (1, 8, 16):
        for out in (BF16, F16):
            assert torch.equal(columns(lambda x: matrix(x, dtype=out), dtype, m), w.float().to(out))
    experts = sw().W4Experts(q.view(3, N // 3, -1), s.view(3, N // 3, -1), z.view(3, N // 3, -1) if zeros else None, group=GROUP)
    for e in range(3):
        ids = torch.full((32, 1), e, dtype=torch.int32, device="cuda")
        one = torch.ones(32, 1, device="cuda")
        want = w[e * N // 3:(e + 1) * N // 3].float().to(F16)
        assert torch.equal(columns(lambda x: experts(x, ids, dtype=F16), dtype, 32), want)
        assert torch.equal(columns(lambda x: experts(x, ids, weights=one, dtype=F16), dtype, 32), want)
    binding.strassen_device_status()


def check_beyond_16_rows(dtype, scales, zeros):
    """Each weight is rounded once, to bf16 beside bf16 rows and to 11 bits beside f16 and e4m3 rows, whatever its group's scale; all
    shapes of the tile kernel: split inner dimension, pairs of CTAs, rows in order of their experts."""
    rounded = BF16 if dtype == BF16 else F16
    for rows, m in ((N, 17), (N, 128), (6500, 512)):
        q, s, z, w = wide_weights(zeros, scales, 2, rows)
        matrix = sw().W4Matrix(q, s, z, group=GROUP)
        x = torch.eye(K, device="cuda").to(dtype)
        parts = [x[i:i + m] if K - i >= m else torch.cat([x[i:], x[:m - K + i]]) for i in range(0, K, m)]
        got = torch.cat([matrix(p, dtype=F16) for p in parts])[:K].t()
        assert torch.equal(got, w.float().to(rounded).to(F16))
    q, s, z, w = wide_weights(zeros, scales, 3)
    experts = sw().W4Experts(q.view(3, N // 3, -1), s.view(3, N // 3, -1), z.view(3, N // 3, -1) if zeros else None, group=GROUP)
    for e in range(3):
        ids = torch.full((128, 1), e, dtype=torch.int32, device="cuda")
        one = torch.ones(128, 1, device="cuda")
        want = w[e * N // 3:(e + 1) * N // 3].float().to(rounded).to(F16)
        assert torch.equal(columns(lambda x: experts(x, ids, dtype=F16), dtype, 128), want)
        assert torch.equal(columns(lambda x: experts(x, ids, weights=one, dtype=F16), dtype, 128), want)
    binding.strassen_device_status()


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("scales", [BF16, F16])
@pytest.mark.parametrize("dtype", [F16, E4M3])
def test_beyond_16_rows_beside_f16_and_e4m3_rows(dtype, scales, zeros):
    check_beyond_16_rows(dtype, scales, zeros)


@pytest.mark.parametrize("zeros", [False, True])
def test_beyond_16_rows_beside_bf16_rows(zeros):
    check_beyond_16_rows(BF16, BF16, zeros)


@pytest.mark.parametrize("zeros", [False, True])
def test_beyond_16_rows_f16_scales_beside_bf16_rows(zeros):
    check_beyond_16_rows(BF16, F16, zeros)
