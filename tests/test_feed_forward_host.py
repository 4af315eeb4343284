"""Host side of the feed-forward operators: the layout's sizes and refusals that need no device."""
import pytest

from paper_1202_3173_b200 import StrassenError, binding


def test_layout_sizes():
    for n, k, group, zeros in ((1, 1, 128, False), (128, 128, 128, True), (129, 257, 32, True), (4096, 12345, 64, False)):
        h = binding.strassen_w4_create(n, k, group, binding.STRASSEN_BF16, zeros)
        tiles = -(-n // 128) * -(-k // 128)
        tile = 8192 + 128 // group * 128 * (3 if zeros else 2)          # nibbles, 16-bit scales, zero points
        assert binding.strassen_w4_bytes(h) == -(-tiles * tile // 256) * 256 + -(-n // 128) * 512
        binding.strassen_w4_destroy(h)


@pytest.mark.parametrize("n,k,group,scale_type", [(0, 1, 32, 0), (1, 0, 32, 0), (-5, 1, 32, 0), (1, 1, 16, 0), (1, 1, 256, 0), (1, 1, 0, 0), (1, 1, 32, 2),
                                                  (1, 1, 32, 3), (1, 1, 32, -1), (2 ** 30 + 1, 1, 32, 0), (2 ** 30, 2 ** 30, 32, 0)])
def test_create_refuses(n, k, group, scale_type):
    with pytest.raises(StrassenError) as e:
        binding.strassen_w4_create(n, k, group, scale_type, False)
    assert e.value.status == -1 and str(e.value)


def test_destroy_takes_null_and_bytes_of_null_are_zero():
    binding.strassen_w4_destroy(None)
    assert binding.strassen_w4_bytes(None) == 0


def test_arguments_are_checked_before_any_device_is_touched():
    for call in (lambda: binding.strassen_rms_norm_quant(-1, 8, 0, 0, 8, 0, 0, 0, 1e-6, 0, 0, 0, 8, 0),
                 lambda: binding.strassen_rms_norm_quant(1, 8, 0, 0, 8, 0, 0, 0, 1e-6, 0, 0, 0, 8, 0),
                 lambda: binding.strassen_silu_mul_quant(1, 8, 7, 256, 8, 256, 8, 4096, 8, 8192),
                 lambda: binding.strassen_silu_mul_quant(1, 8, 0, 256, 8, 0, 8, 4096, 8, 8192),
                 lambda: binding.strassen_w4_matmul(0, 1, 0, 256, 8, 0, 0, 4096, 8)):
        with pytest.raises(StrassenError) as e:
            call()
        assert e.value.status == -1 and str(e.value)


def test_the_package_offers_the_operators():
    import paper_1202_3173_b200 as sw
    for name in ("W4Matrix", "FeedForward", "rms_norm_quant", "silu_mul_quant", "quant_rows"):
        assert name in sw.__all__ and callable(getattr(sw, name))
    with pytest.raises(AttributeError):
        sw.no_such_operator
