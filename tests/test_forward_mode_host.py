"""Forward-mode tangents are refused by the operators of a served model, before anything else is looked at: they have no derivatives, and would drop them without a word."""
import pytest
import torch
from torch.autograd import forward_ad

import paper_1202_3173_b200 as sw


def dual(*shape, dtype=torch.bfloat16):
    x = torch.ones(*shape, dtype=dtype)
    return forward_ad.make_dual(x, torch.ones_like(x))


def plain(*shape, dtype=torch.bfloat16):
    return torch.ones(*shape, dtype=dtype)


CALLS = {
    "norm, x": lambda t: sw.rms_norm_quant(t(2, 64), plain(64)),
    "norm, weight": lambda t: sw.rms_norm_quant(plain(2, 64), t(64)),
    "norm, residual": lambda t: sw.rms_norm_quant(plain(2, 64), plain(64), residual=t(2, 64)),
    "norm, sum": lambda t: sw.rms_norm_quant(plain(2, 64), plain(64), residual=plain(2, 64), out=(plain(2, 64), plain(2), t(2, 64))),
    "gate": lambda t: sw.silu_mul_quant(t(2, 64), plain(2, 64)),
    "up": lambda t: sw.silu_mul_quant(plain(2, 64), t(2, 64)),
    "routing": lambda t: sw.route_experts(t(2, 8), 2),
    "routing, bias": lambda t: sw.route_experts(plain(2, 8), 2, bias=t(8, dtype=torch.float32)),
    "matrix": lambda t: sw.W4Matrix(torch.zeros(8, 32, dtype=torch.uint8), t(8, 1), group=64),
    "experts": lambda t: sw.W4Experts(torch.zeros(2, 8, 32, dtype=torch.uint8), t(2, 8, 1), group=64),
    "storing, q": lambda t: sw.rotate_append(t(2, 4, 64), plain(2, 2, 64), plain(2, 2, 64), None, None, None),
    "storing, k": lambda t: sw.rotate_append(plain(2, 4, 64), t(2, 2, 64), plain(2, 2, 64), None, None, None),
    "storing, v": lambda t: sw.rotate_append(plain(2, 4, 64), plain(2, 2, 64), t(2, 2, 64), None, None, None),
    "storing, frequencies": lambda t: sw.rotate_append(None, plain(2, 2, 64), plain(2, 2, 64), None, None, None, t(32, dtype=torch.float32)),
    "one token": lambda t: sw.decode_attention(t(2, 4, 64), None, None, None),
    "one token, out": lambda t: sw.decode_attention(plain(2, 4, 64), None, None, None, out=t(2, 4, 64)),
    "prompts": lambda t: sw.prompt_attention(t(2, 4, 64), None, None, None, plain(2)),
    "cache": lambda t: sw.PagedCache(t(2, 2, 16, 64), plain(2, 2, 16, 64)),
}


@pytest.mark.parametrize("name", CALLS)
def test_tangents_are_refused(name):
    with forward_ad.dual_level():
        with pytest.raises(ValueError, match="tangent"):
            CALLS[name](dual)
        # others go on to the next check, which is that of devices here
        with pytest.raises((ValueError, AttributeError)) as e:
            CALLS[name](plain)
        assert "tangent" not in str(e.value)


def test_products_of_laid_out_matrices():
    for kind in (sw.W4Matrix, sw.W4Experts):
        m = kind.__new__(kind)
        m._h = 1
        try:
            args = (torch.zeros(2, 1, dtype=torch.int32),) if kind is sw.W4Experts else ()
            with forward_ad.dual_level():
                for change in (dict(x=dual(2, 64)), dict(x_scale=dual(2, dtype=torch.float32)), dict(out=dual(2, 8))):
                    with pytest.raises(ValueError, match="tangent"):
                        m(change.pop("x", plain(2, 64)), *args, **change)
        finally:
            m._h = None
