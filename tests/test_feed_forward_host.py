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


@pytest.mark.parametrize("experts", [0, -1, 1025])
def test_create_refuses_experts(experts):
    with pytest.raises(StrassenError) as e:
        binding.strassen_w4_create_experts(experts, 16, 16, 32, 0, False)
    assert e.value.status == -1 and str(e.value)


def test_experts_are_laid_out_one_after_another():
    one, many = binding.strassen_w4_create(200, 300, 64, 0, True), binding.strassen_w4_create_experts(5, 200, 300, 64, 0, True)
    tile = 8192 + 2 * 128 * 3
    assert binding.strassen_w4_bytes(one) == -(-2 * 3 * tile // 256) * 256 + 2 * 512
    assert binding.strassen_w4_bytes(many) == -(-5 * 2 * 3 * tile // 256) * 256 + 5 * 2 * 512
    assert binding.strassen_w4_experts_workspace_bytes(many, 4, 8, True) == 0
    assert binding.strassen_w4_experts_workspace_bytes(many, 5, 8, True) - binding.strassen_w4_experts_workspace_bytes(many, 5, 8, False) == 40 * 200 * 4
    for h in (one, many):
        binding.strassen_w4_destroy(h)


def test_routing_arguments_are_checked_before_any_device_is_touched():
    ok = dict(tokens=1, experts=64, type=2, logits=4096, ld=64, bias=0, score=0, groups=8, top_groups=4, top=8, renormalize=True, factor=1.0, ids=8192, weights=12288)
    for change in (dict(tokens=-1), dict(experts=0), dict(experts=1025), dict(type=3), dict(score=2), dict(groups=0), dict(groups=7), dict(groups=64),
                   dict(top_groups=0), dict(top_groups=9), dict(top=0), dict(top=33), dict(top_groups=1, top=9), dict(factor=float("nan")), dict(logits=0), dict(ids=0), dict(weights=0)):
        with pytest.raises(StrassenError) as e:
            binding.strassen_route_experts(**{**ok, **change})
        assert e.value.status == -1, change
    for status, change in ((-5, dict(logits=4098)), (-5, dict(ids=8193)), (-5, dict(bias=2)), (-4, dict(ids=4096)), (-4, dict(weights=8192))):
        with pytest.raises(StrassenError) as e:
            binding.strassen_route_experts(**{**ok, **change})
        assert e.value.status == status, change


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
    for name in ("W4Matrix", "W4Experts", "FeedForward", "ExpertsFeedForward", "rms_norm_quant", "silu_mul_quant", "route_experts", "quant_rows"):
        assert name in sw.__all__ and callable(getattr(sw, name))
    with pytest.raises(AttributeError):
        sw.no_such_operator
