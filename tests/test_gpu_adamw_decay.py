"""A state's weight decays may be set between steps."""
import math

import pytest
import torch

import paper_2605_03667_amd as elas

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_decays_that_are_set():
    """A step without a gradient, of moments that are 0, takes rate * decay of a weight off it (1 - 2^-4 d and its product
    are exact here)."""
    params = [torch.ones(300, device=DEV), torch.ones(5, device=DEV)]
    opt = elas.ElasAdamW(params, decay=[1.0, 0.0])
    grads = [torch.zeros_like(p) for p in params]
    elas.elas_adamw_step(opt, grads, 0.0625)
    assert (params[0] == 0.9375).all() and (params[1] == 1).all()
    opt.decay = [0.0, 2.0]
    assert list(opt.decay) == [0.0, 2.0]
    elas.elas_adamw_step(opt, grads, 0.0625)
    assert (params[0] == 0.9375).all() and (params[1] == 0.875).all()
    opt.decay = 8.0
    assert list(opt.decay) == [8.0, 8.0]
    elas.elas_adamw_step(opt, grads, 0.0625)
    assert (params[0] == 0.46875).all() and (params[1] == 0.4375).all()
    # one decay is not set by itself, without the state's knowing
    with pytest.raises(TypeError):
        opt.decay[0] = 1.0
    for bad, match in (([1.0], "1 decays"), ([1.0, math.inf], "finite"), (math.nan, "finite")):
        with pytest.raises(ValueError, match=match):
            opt.decay = bad
    elas.elas_adamw_step(opt, grads, 0.0625)
    assert (params[0] == 0.234375).all()
