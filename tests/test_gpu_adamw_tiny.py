"""Moments in 8 bits whose block's scale is below float32's normal range: codes that stand for the
moments all the same."""
import pytest
import torch

import paper_2605_03667_amd as elas

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
SMALLEST = 2.0 ** -149          # float32's


def _gradient(size, n=1024):
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    sign = torch.where(torch.rand(n, generator=g, device=DEV) < 0.5, -1.0, 1.0)
    return sign * (0.5 + 0.5 * torch.rand(n, generator=g, device=DEV)) * size


def _pair(grad):
    """The same first step with moments in 32 and in 8 bits, at a rate of 0."""
    opts = [elas.ElasAdamW([torch.zeros_like(grad)], bits=bits) for bits in (32, 8)]
    for opt in opts:
        elas.elas_adamw_step(opt, [grad], 0.0, beta1=0.9, beta2=0.95, eps=1e-30)
    return opts


# (first moments of a tenth of that, second ones of a twentieth of its square)
@pytest.mark.parametrize("size", [1e-43, 3e-42, 1e-39, 1.7e-38, 2.3e-38, 1e-37, 1e-22, 1e-21, 1e-20, 1.2e-19, 1.7e-19, 2.1e-19, 5e-19, 1e-17])
def test_codes_stand_for_small_moments(size):
    """What is rounded are the moments of 32 bits (the arithmetic is the same), each to one of the two codes beside it: at
    most 2^-3 of itself away (second ones 2^-4), or a unit of the scale where it is below 2^3 (2^4) units.  The scale is the largest
    magnitude's over the largest code, to 2 roundings, or at most a step of 2^-149 above it; reading a code out rounds once more."""
    wide, eight = _pair(_gradient(size))
    for name, mantissa, top in (("m", 3, 245760.0), ("v", 4, 507904.0)):
        x = getattr(wide, name).double().abs()
        got = elas.elas_adam8_values(getattr(eight, name), getattr(eight, name + "_scale"), second=name == "v", dtype=torch.float32).double().abs()
        unit = (x.view(-1, 256).amax(1, keepdim=True) / top * (1 + 2.0 ** -23) + SMALLEST).expand(-1, 256).reshape(-1)
        near = x * (2.0 ** -mantissa + 2.0 ** -22) + unit + SMALLEST
        assert ((got - x).abs() <= near).all(), (name, size, ((got - x).abs() / near).max())
        if name == "v":
            assert ((got > 0) == (x > 0)).all()


@pytest.mark.parametrize("size", [1e-20, 1.2e-19, 1.7e-19, 1e-18])
def test_the_next_step_from_small_moments(size):
    """A step without a gradient moves a weight by the rate times the moments' ratio.  The first moment is off by at most 1/8 of
    itself, the second by 1/16, of whose smallest (a quarter of 5e-42, 890 steps of 2^-149) fading and reading out round
    half a step each: 2^-9 in all of the ratio."""
    grad = _gradient(size)
    opts = _pair(grad)
    for opt in opts:
        elas.elas_adamw_step(opt, [torch.zeros_like(grad)], 1.0, beta1=0.9, beta2=0.95, eps=1e-30)
    wide, eight = (opt.params.tensors[0].double() for opt in opts)
    ratio = eight / wide
    assert torch.isfinite(ratio).all()
    assert ratio.min() >= (1 - 1 / 8) / (1 + 1 / 16) ** 0.5 * (1 - 2.0 ** -9)
    assert ratio.max() <= (1 + 1 / 8) / (1 - 1 / 16) ** 0.5 * (1 + 2.0 ** -9)
