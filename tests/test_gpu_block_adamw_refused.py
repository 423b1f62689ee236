"""A step over ring stores that is refused: the layers' shards have not been brought home for it."""
import math

import pytest
import torch

from paper_2311_01635_amd import RtpAdamW
from paper_2311_01635_amd import binding as B
from paper_2311_01635_amd.layers import RtpLinear

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_refused_step_leaves_the_stores_as_they_are():
    n, T, I, O = 4, 32, 64, 128
    g = torch.Generator().manual_seed(0)
    layer = RtpLinear(torch.randn(O, I, generator=g) * 0.05, T, n, 1)
    opt = RtpAdamW.for_layers([layer])
    X, dY = (torch.randn(T, w, generator=g).to(DEV, torch.bfloat16) for w in (I, O))
    Y, dX = torch.empty_like(dY), torch.empty_like(X)
    layer.forward(X, Y)
    layer.backward(X, dY, dX)
    layer.sync()
    before = layer.home_w.clone(), layer.home_g.clone()
    off = torch.zeros(128, dtype=torch.uint8, device=DEV)
    off[8:56] = RtpAdamW.scalars_of(1e-3, 1).to(DEV)
    for kw in (dict(lr=math.nan, step=1), dict(lr=1e-3, step=0), dict(lr=1e-3, step=1, betas=(0.9, 1.0)), dict(lr=1e-3, step=1, eps=0.0),
               dict(lr=None, step=None, scalars=off[8:56])):
        with pytest.raises((B.RtpError, ValueError)):
            opt.step(**kw)
        layer.sync()
        assert torch.equal(before[0], layer.home_w) and torch.equal(before[1], layer.home_g), kw
    opt.step(1e-3, 1)
    layer.sync()
    torch.cuda.synchronize()
    assert not torch.equal(before[0], layer.home_w) and (layer.home_g == 0).all()
    opt.close()
    layer.forward(X, Y)
    layer.backward(X, dY, dX)
    layer.sync()
    before = layer.home_w.clone(), layer.home_g.clone()
    with pytest.raises(B.RtpError):
        opt.step(1e-3, 2)                                     # closed
    layer.sync()
    assert torch.equal(before[0], layer.home_w) and torch.equal(before[1], layer.home_g)
    layer.close()
