"""Gradient of sigmoid scores near 1: the factor 1 - s, relative to itself.

u = 2^-24.  1 - s = 1 / (1 + e^x): an exponential (2 u), a sum and a quotient.  Not renormalised, three products on top and the sigmoid
itself: 16 u of the entry.  Renormalised, w_j (1 - s_j) (a_j - sum w_i a_i / scale): what is subtracted is off by (2 k + 16) u of the largest
|a|, everything else by as much of itself."""
import pytest
import torch

from paper_2311_01635_amd import RtpRouter

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E,k", [(8, 2), (64, 6), (512, 8)])
def test_gradient_of_strongly_chosen_experts(E, k, renorm):
    g = torch.Generator().manual_seed(E)
    T, scale = 128, 2.5
    l = 10 + 50 * torch.rand(T, E, generator=g)
    ids, w = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
    r = RtpRouter(E, k, score="sigmoid", renormalise=renorm, scale=scale)
    r.forward(l.to(DEV), ids, w)
    a = torch.randn(T, k, generator=g)
    dl = torch.full((T, E), float("nan"), device=DEV)
    r.backward(l.to(DEV), ids, a.to(DEV), dl)
    ids, a = ids.cpu().long(), a.double()
    x = l.double().gather(1, ids)
    s, rest = 1 / (1 + torch.exp(-x)), 1 / (1 + torch.exp(x))
    if renorm:
        q = s / s.sum(1, keepdim=True)
        want = scale * q * rest * (a - (q * a).sum(1, keepdim=True))
        tol = scale * q * rest * (2 * k + 16) * U * (a.abs() + a.abs().amax(1, keepdim=True))
    else:
        want = scale * s * rest * a
        tol = 16 * U * want.abs()
    assert float(want.abs().min()) < 1e-20                    # (far below what 1 - s leaves of them)
    assert ((dl.cpu().double().gather(1, ids) - want).abs() <= tol).all()
    chosen = torch.zeros(T, E, dtype=torch.bool).scatter_(1, ids, True)
    assert (dl.cpu()[~chosen] == 0).all()
