"""Offsets past 32 bits: rows, slots and parameters that lie more than 2^32 bytes (and 2^31 elements) from the first, against the same
values close together.  Only the rows themselves are touched."""
import math

import pytest
import torch

from paper_2311_01635_amd import RtpAdamW, RtpCombine, RtpNorm, RtpRouter

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LD = 1 << 28                 # elements from row to row
F32, BF16 = torch.float32, torch.bfloat16


def _far(t):
    """t's rows, LD elements apart"""
    big = torch.empty((t.shape[0] - 1) * LD + t.shape[1], dtype=t.dtype, device=DEV)
    v = big.as_strided(t.shape, (LD, 1))
    v.copy_(t)
    return v


@pytest.mark.parametrize("D", [136, 4097, 20000])
def test_norm(D):
    T = 10                   # 2.4e9 elements
    g = torch.Generator(device=DEV).manual_seed(D)
    rnd = lambda: torch.randn(T, D, generator=g, device=DEV).to(BF16)   # noqa: E731
    n = RtpNorm(D, kind="layer", post=True, w_post=torch.ones(D, device=DEV), w_pre=torch.ones(D, device=DEV))
    x, y, gate, dr, dh = (rnd() for _ in range(5))
    out = []
    for place in (lambda t: t, _far):
        new = lambda: place(torch.full((T, D), math.nan, dtype=BF16, device=DEV))   # noqa: E731
        r, h, dx, dy, dg, st = new(), new(), new(), new(), new(), torch.empty(T, 4, device=DEV)
        n.forward(place(x), place(y), r, h, st, gate=place(gate))
        w = n.backward(r, place(y), place(dr), place(dh), dx, dy, st, gate=place(gate), dgate=dg, accumulate=False)
        out.append([t.clone() for t in (r, h, dx, dy, dg, st, *w.values())])
        del r, h, dx, dy, dg
        torch.cuda.empty_cache()
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_combine():
    T, k, D = 5, 2, 520
    g = torch.Generator(device=DEV).manual_seed(1)
    yk, dy, w = torch.randn(T * k, D, generator=g, device=DEV).to(BF16), torch.randn(T, D, generator=g, device=DEV).to(BF16), torch.rand(T, k, generator=g, device=DEV)
    c, out = RtpCombine(k), []
    for place in (lambda t: t, _far):
        Y, dyk, dw = place(torch.zeros_like(dy)), place(torch.zeros_like(yk)), torch.empty(T, k, device=DEV)
        c.forward(place(yk), w, Y)
        c.backward(place(dy), place(yk), w, dyk, dw)
        out.append([t.clone() for t in (Y, dyk, dw)])
    assert all(torch.equal(a, b) for a, b in zip(*out))


def test_router():
    T, E, k = 10, 40, 4
    l = torch.randn(T, E, device=DEV)
    r, out = RtpRouter(E, k, bias=0.1 * torch.randn(E, device=DEV)), []
    for place in (lambda t: t, _far):
        ids, w, dl = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV), place(torch.zeros(T, E, device=DEV))
        r.forward(place(l), ids, w)
        r.backward(place(l), ids, w, dl)
        out.append([t.clone() for t in (ids, w, dl)])
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("state", ["f32", "8bit"])
def test_adamw(state):
    """one tensor of more than 2^31 elements: its end against a tensor of that end alone"""
    n, tail = (1 << 31) + 4096 * 3 + 77, 4096 + 77
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    at = n - tail            # (a whole number of blocks)
    assert at % 256 == 0
    gen = torch.Generator(device=DEV).manual_seed(2)
    p[at:], g[at:] = torch.randn(tail, generator=gen, device=DEV), torch.randn(tail, generator=gen, device=DEV)
    q, h = p[at:].clone(), g[at:].clone()
    big, small = RtpAdamW([dict(param=p, grad=g, weight_decay=0.1)], state), RtpAdamW([dict(param=q, grad=h, weight_decay=0.1)], state)
    for opt in (big, small):
        opt.step(1e-2, 1)    # (from zeros: an fp32 parameter's first step has no rounding at random in it)
    assert torch.equal(p[at:], q) and float((q - p[at:]).abs().max()) == 0 and float(q.abs().max()) > 0
    assert float(p[:at].abs().max()) == 0
    if state == "f32":
        assert torch.equal(big.m[at:at + tail], small.m[:tail]) and torch.equal(big.v[at:at + tail], small.v[:tail])
    else:
        assert torch.equal(big.exps[at // 256:], small.exps)
