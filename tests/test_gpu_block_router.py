"""Router and combination against their definitions in 64 bits.

Tolerances.  u = 2^-24 is half an fp32 step.  An exponential of l - m carries the rounding of its argument, |l - m| u of the
value, and one of its own; a sum of n positive numbers at most n u; so a weight is within (R + 2 k + 12) u of itself, R the
largest |l - m| (and of log sigmoid, which is as large).  16-bit outputs: half a step of the type on top."""
import math
import random

import pytest
import torch

import block_reference as ref
from paper_2311_01635_amd import RtpCombine, RtpRouter

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
CASES = [  # T, E, k, kwargs
    (1, 1, 1, dict()), (1, 8, 2, dict()), (37, 8, 8, dict(score="sigmoid")), (300, 64, 6, dict(renorm=False)), (5, 3, 1, dict(renorm=False, scale=0.5)),
    (129, 160, 6, dict(groups=8, kept=3, group_top=1)), (64, 256, 8, dict(score="sigmoid", groups=8, kept=4, group_top=2, scale=2.5)),
    (63, 96, 4, dict(score="sigmoid", groups=32, kept=2, group_top=2)), (33, 60, 7, dict(groups=5, kept=5, group_top=2)), (17, 100, 32, dict(score="sigmoid", renorm=False)),
    (9, 1024, 32, dict()), (9, 1023, 3, dict(score="sigmoid")), (1000, 7, 3, dict()), (3, 64, 12, dict(groups=64, kept=12)), (40, 512, 1, dict()), (21, 33, 5, dict(score="sigmoid", scale=-1.5)),
]


def _logits(T, E, dtype, seed, closed=0.0, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    l = torch.randn(T, E, generator=g) * spread
    if closed:
        l[torch.rand(T, E, generator=g) < closed] = -math.inf
    return l.to(dtype)


def _run(l, k, bias=None, ids_T=None, **kw):
    kw = dict(kw)
    r = RtpRouter(l.shape[1], k, score=kw.get("score", "softmax"), renormalise=kw.get("renorm", True), scale=kw.get("scale", 1.0), groups=kw.get("groups", 1),
                  kept_groups=kw.get("kept", 1), group_top=kw.get("group_top", 1), bias=bias)
    ids, w = torch.full((l.shape[0], k), -7, dtype=torch.int32, device=DEV), torch.full((l.shape[0], k), math.nan, device=DEV)
    r.forward(l, ids, w)
    return r, ids, w


def _tol(l, k):
    f = l.double()[l > -math.inf]
    R = float(f.abs().max()) * 2 if f.numel() else 0.0
    return (R + 2 * k + 12) * U


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:3])))
def test_forward(case, biased, dtype):
    T, E, k, kw = case
    for closed in (0.0, 0.3):
        l = _logits(T, E, dtype, T * 7 + E, closed)          # (16-bit logits hold equal ones: the lowest index first)
        bias = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(E)) if biased else None
        _, ids, w = _run(l.to(DEV), k, None if bias is None else bias.to(DEV), **kw)
        want_ids, want_w = ref.route(l, k, bias=bias, **kw)
        assert torch.equal(ids.cpu(), want_ids)
        err = (w.cpu().double() - want_w).abs()
        assert (err <= _tol(l, k) * want_w.abs()).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("groups", [1, 4])
def test_closed_rows_and_lowest_values(score, renorm, groups):
    kw = dict(score=score, renorm=renorm, groups=groups, kept=min(groups, 2), group_top=2)
    T, E, k = 12, 32, 5
    l = _logits(T, E, F32, 3)
    l[0] = -math.inf                                          # no expert is open
    l[1] = -math.inf
    l[1, 9] = 0.5                                             # one is
    l[2, 4:] = torch.finfo(F32).min                           # a mask of the type's lowest value: open, but last
    l[3] = torch.finfo(F32).min
    l[4] = -300.0                                             # sigmoids that underflow
    l[5] = 200.0
    l[6] = 1e30
    for bias in (None, torch.linspace(-1, 1, E)):
        r, ids, w = _run(l.to(DEV), k, None if bias is None else bias.to(DEV), **kw)
        want_ids, want_w = ref.route(l, k, bias=bias, **kw)
        assert torch.equal(ids.cpu(), want_ids)
        assert (w[0] == 0).all() and (w[1, 1:] == 0).all() and w[1, 0] > 0
        # (a sigmoid that is not renormalised may be a denormal: to the smallest of fp32)
        rows = [0, 1, 2, 7, 8, 9, 10, 11] if not renorm else list(range(12))
        assert ((w.cpu().double() - want_w).abs() <= (800 + 2 * k) * U * want_w.abs() + 2.0 ** -149)[rows].all()
        dl = torch.full((T, E), math.nan, device=DEV)
        dw = torch.randn(T, k, generator=torch.Generator().manual_seed(1)).to(DEV)
        dw[0] = math.nan                                      # a closed slot's output was not looked at: its gradient has no part
        dw[1, 1:] = math.inf
        r.backward(l.to(DEV), ids, dw, dl)
        assert (dl[0] == 0).all() and torch.isfinite(dl).all()
        assert (dl.cpu()[l == -math.inf] == 0).all()


def test_nan_shows_and_stays_in_its_row():
    l = _logits(6, 16, F32, 5)
    l[2, 11] = math.nan
    for score in ("softmax", "sigmoid"):
        for groups in (1, 4):
            r, ids, w = _run(l.to(DEV), 4, score=score, groups=groups, kept=2 if groups > 1 else 1)
            assert torch.isnan(w[2]).any() and torch.isfinite(w[[0, 1, 3, 4, 5]]).all()
            i = ids.cpu()
            assert ((i >= 0) & (i < 16)).all() and all(len(set(x)) == 4 for x in i.tolist())
            dl = torch.empty(6, 16, device=DEV)
            r.backward(l.to(DEV), ids, torch.ones(6, 4, device=DEV), dl)
            assert torch.isfinite(dl[[0, 1, 3, 4, 5]]).all() and torch.isnan(dl[2]).any()


def test_near_ties_are_decided_in_64_bits():
    """two choices that are one fp32 number apart in neither term: the bias decides by less than 2^-24"""
    E = 64
    l = torch.zeros(8, E)
    bias = torch.zeros(E)
    bias[37] = 2.0 ** -40
    bias[5] = 2.0 ** -41
    _, ids, _ = _run(l.to(DEV), 3, bias.to(DEV), score="sigmoid")
    assert ids.cpu().tolist() == [[37, 5, 0]] * 8


@pytest.mark.parametrize("seed", range(40))
def test_configurations(seed):
    """any number of experts, groups and choices together"""
    r = random.Random(seed)
    groups = r.choice([1, 2, 3, 4, 7, 8, 16, 33, 64])
    E = groups * r.randint(1, max(1, (16, 64, 256, 1024)[seed % 4] // groups))
    kept = r.randint(1, groups)
    k = r.randint(1, min(32, E // groups * kept))
    kw = dict(score=r.choice(["softmax", "sigmoid"]), renorm=r.random() < 0.5, scale=r.choice([1.0, 2.5]), groups=groups, kept=kept, group_top=r.choice([1, 2]))
    dtype = r.choice([F32, BF16, F16])
    T = r.randint(1, 70)
    l = _logits(T, E, dtype, seed, closed=r.choice([0.0, 0.5, 0.97]))
    bias = 0.1 * torch.randn(E, generator=torch.Generator().manual_seed(seed)) if r.random() < 0.5 else None
    _, ids, w = _run(l.to(DEV), k, None if bias is None else bias.to(DEV), **kw)
    want_ids, want_w = ref.route(l, k, bias=bias, **kw)
    assert torch.equal(ids.cpu(), want_ids), (T, E, k, kw)
    assert ((w.cpu().double() - want_w).abs() <= (_tol(l, k) + (E / 64 + 16) * U) * want_w.abs()).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("E,groups", [(32, 4), (256, 8), (600, 6)])
def test_choices_about_as_close_as_32_bits_can_tell(E, groups, biased, score):
    """scores and biases that differ by 2^-16 to 2^-26 of themselves, around several sizes: whichever of them the kernel decides in 32 bits, it
    decides as 64 bits do"""
    g = torch.Generator().manual_seed(E)
    T = 96
    size = torch.tensor([0.0, 1.0, -3.0, 6.0, -20.0, 12.0])[torch.arange(T) % 6][:, None]
    spread = 2.0 ** -torch.randint(16, 27, (T, 1), generator=g)
    l = size * (1 + spread * torch.randn(T, E, generator=g)) + spread * torch.randn(T, E, generator=g)
    bias = 1.0 + 2.0 ** -20 * torch.randn(E, generator=g) if biased else None
    # (equal logits with equal biases are equal in any arithmetic; others differ by 2^-24 of something, where 64 bits have 2^-52 left)
    _, ids, _ = _run(l.to(DEV), 6, None if bias is None else bias.to(DEV), score=score, groups=groups, kept=3)
    assert torch.equal(ids.cpu(), ref.route(l, 6, score=score, groups=groups, kept=3, bias=bias)[0])


@pytest.mark.parametrize("gdt", [F32, BF16, F16])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:3])))
def test_backward(case, dtype, gdt):
    T, E, k, kw = case
    l = _logits(T, E, dtype, T + E)
    r, ids, _ = _run(l.to(DEV), k, **kw)
    g = torch.randn(T, k, generator=torch.Generator().manual_seed(2))
    dl = torch.full((T, E), math.nan, device=DEV, dtype=gdt)
    r.backward(l.to(DEV), ids, g.to(DEV), dl)
    leaf = l.double().requires_grad_()
    scale, renorm, score = kw.get("scale", 1.0), kw.get("renorm", True), kw.get("score", "softmax")
    w = ref.route_weights(leaf, ids.cpu(), score, renorm, scale)
    (w * g.double()).sum().backward()
    # every factor is at most 1 but the gradient of the weights and the scale, and what is subtracted at most max |g|
    most = abs(scale) * float(g.abs().max())
    tol = (_tol(l, k) + (E / 64 + 16) * U) * 2 * most + torch.finfo(gdt).eps / 2 * leaf.grad.abs() + (2.0 ** -25 if gdt == F16 else 0)
    assert ((dl.cpu().double() - leaf.grad).abs() <= tol).all()
    # ... and by differences of the 64-bit weights along a direction (central, step 1e-4: truncation 1e-8 of a third derivative below 10)
    d = torch.randn(T, E, generator=torch.Generator().manual_seed(3)).double()
    f = lambda s: (ref.route_weights(l.double() + s * d, ids.cpu(), score, renorm, scale) * g.double()).sum()   # noqa: E731
    slope = float(f(1e-4) - f(-1e-4)) / 2e-4
    slack = float((tol * d.abs()).sum()) + 1e-6 * T * k * most
    assert abs(float((dl.cpu().double() * d).sum()) - slope) <= slack


def test_backward_of_ids_that_name_nothing_and_one_twice():
    T, E, k = 4, 8, 3
    l = _logits(T, E, F32, 0)
    r = RtpRouter(E, k, score="sigmoid", renormalise=False)
    ids = torch.tensor([[0, 1, 2], [3, 3, 4], [-1, 8, 2 ** 31 - 1], [7, 0, -5]], dtype=torch.int32, device=DEV)
    g = torch.ones(T, k, device=DEV)
    dl = torch.full((T, E), math.nan, device=DEV)
    r.backward(l.to(DEV), ids, g, dl)
    s = torch.sigmoid(l.double())
    n = torch.zeros(T, E, dtype=torch.float64)
    n[0, :3] = 1; n[1, 3] = 2; n[1, 4] = 1; n[3, 7] = 1; n[3, 0] = 1     # noqa: E702
    assert ((dl.cpu().double() - n * s * (1 - s)).abs() <= 16 * U * n).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides_offsets_and_rows_behind(dtype):
    T, E, k = 13, 40, 4
    l = _logits(T, E, dtype, 8)
    wide = torch.full((T + 2, E + 7), math.nan, dtype=dtype, device=DEV)
    view = wide[:T, 3:3 + E]
    view.copy_(l)
    r, ids, w = _run(view, k)
    want_ids, want_w = ref.route(l, k)
    assert torch.equal(ids.cpu(), want_ids) and ((w.cpu().double() - want_w).abs() <= _tol(l, k) * want_w).all()
    out = torch.full((T + 2, E + 9), 5.0, dtype=dtype, device=DEV)
    dense = torch.empty(T, E, dtype=dtype, device=DEV)
    g = torch.randn(T, k, device=DEV)
    r.backward(view, ids, g, out[1:T + 1, 1:1 + E])
    r.backward(l.to(DEV), ids, g, dense)
    assert torch.equal(out[1:T + 1, 1:1 + E], dense)
    out[1:T + 1, 1:1 + E] = 5.0
    assert (out == 5.0).all()


def test_many_rows():
    """more rows than a grid has workgroups at once, and an odd number"""
    T, E, k = 70001, 8, 2
    l = torch.randn(T, E, generator=torch.Generator().manual_seed(1))
    _, ids, w = _run(l.to(DEV), k)
    top = l.double().sort(dim=1, descending=True, stable=True)
    assert torch.equal(ids.cpu().long(), top.indices[:, :k])
    want = torch.softmax(top.values[:, :k], 1)
    assert ((w.cpu().double() - want).abs() <= _tol(l, k) * want).all()


# ---- combination ------------------------------------------------------------------------------------------------------

SHAPES = [(1, 1, 1), (1, 8, 7), (5, 2, 64), (33, 3, 1000), (129, 8, 768), (7, 32, 513), (64, 2, 4096), (3, 4, 8193), (2, 1, 20000), (1000, 2, 16)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_combine(shape, dtype):
    T, k, D = shape
    g = torch.Generator().manual_seed(T + D)
    yk, dy = torch.randn(T * k, D, generator=g).to(dtype), torch.randn(T, D, generator=g).to(dtype)
    w = torch.rand(T, k, generator=g)
    w[torch.rand(T, k, generator=g) < 0.2] = 0.0
    yk[(w == 0).view(-1)] = math.nan                          # what a slot without weight holds is not looked at
    Y = torch.full((T, D), math.nan, dtype=dtype, device=DEV)
    c = RtpCombine(k)
    c.forward(yk.to(DEV), w.to(DEV), Y)
    y64 = torch.where((w == 0)[:, :, None], 0.0, yk.double().view(T, k, D))
    want, size = (w.double()[:, :, None] * y64).sum(1), (w.double()[:, :, None] * y64.abs()).sum(1)
    half = torch.finfo(dtype).eps / 2
    tiny = 2.0 ** -25 if dtype == F16 else 0
    assert ((Y.cpu().double() - want).abs() <= half * want.abs() * 1.01 + (k + 1) * U * size + tiny).all()
    dyk, dw = torch.full((T * k, D), math.nan, dtype=dtype, device=DEV), torch.full((T, k), math.nan, device=DEV)
    c.backward(dy.to(DEV), yk.to(DEV), w.to(DEV), dyk, dw)
    want = (w.double()[:, :, None] * dy.double()[:, None]).view(T * k, D)
    assert ((dyk.cpu().double() - want).abs() <= half * want.abs() + tiny).all()
    prod = dy.double()[:, None] * y64
    err = (dw.cpu().double() - prod.sum(2)).abs()
    # (a sum of D products: each lane adds D / 64 of them at most, then the lanes')
    assert (err <= (D / 64 + 16) * U * prod.abs().sum(2))[w != 0].all()
    only = torch.full((T, k), math.nan, device=DEV)
    c.backward(dy.to(DEV), yk.to(DEV), w.to(DEV), None, only)
    assert torch.equal(only.cpu()[w != 0], dw.cpu()[w != 0])
    # expansion, and its gradient
    c.expand(dy.to(DEV), dyk)
    assert torch.equal(dyk.cpu(), dy.repeat_interleave(k, 0))
    c.forward(dyk, None, Y)
    want = k * dy.double()
    assert ((Y.cpu().double() - want).abs() <= half * want.abs() * 1.01 + (k + 1) * U * want.abs() + tiny).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("off,pad", [(0, 8), (1, 3), (3, 0)])
def test_combine_strides(off, pad, dtype):
    """columns that start off 16 bytes, rows that are apart; what lies between stays"""
    T, k, D = 9, 3, 136
    g = torch.Generator().manual_seed(0)

    def view(rows):
        t = torch.full((rows + 1, D + off + pad), 3.0, dtype=dtype, device=DEV)
        return t, t[:rows, off:off + D]
    yk, Y, dY, dYk = view(T * k), view(T), view(T), view(T * k)
    yk[1].copy_(torch.randn(T * k, D, generator=g))
    dY[1].copy_(torch.randn(T, D, generator=g))
    w = torch.rand(T, k, generator=g).to(DEV)
    c = RtpCombine(k)
    c.forward(yk[1], w, Y[1])
    plain = torch.empty(T, D, dtype=dtype, device=DEV)
    c.forward(yk[1].contiguous(), w, plain)
    assert torch.equal(plain, Y[1])
    dw, dw2, plain = torch.empty(T, k, device=DEV), torch.empty(T, k, device=DEV), torch.empty(T * k, D, dtype=dtype, device=DEV)
    c.backward(dY[1], yk[1], w, dYk[1], dw)
    c.backward(dY[1].contiguous(), yk[1].contiguous(), w, plain, dw2)
    # (rows off 16 bytes may be summed in another order)
    size = (dY[1].double()[:, None] * yk[1].double().view(T, k, D)).abs().sum(2)
    assert torch.equal(plain, dYk[1]) and ((dw - dw2).abs() <= 2 * (D / 64 + 16) * U * size).all()
    for t, v in (Y, dYk):
        v.fill_(3.0)
        assert (t == 3.0).all()


def test_refusals_on_the_device():
    r, i, w = RtpRouter(8, 2), torch.empty(4, 2, dtype=torch.int32, device=DEV), torch.empty(4, 2, device=DEV)
    l = torch.zeros(4, 8, device=DEV)
    for bad in ((l.double(), i, w), (l[:, :7], i, w), (l, i.long(), w), (l, i[:3], w), (l, i, w.half()), (l, i, w[:, :1]), (l.t().contiguous().t(), i, w),
                (l[:1].expand(4, 8), i, w), (l[0], i, w)):
        with pytest.raises(ValueError):
            r.forward(*bad)
    with pytest.raises(ValueError):
        r.backward(l, i, w, torch.empty(4, 8, device=DEV, dtype=torch.float64))
    with pytest.raises(ValueError):
        RtpRouter(8, 2, bias=torch.zeros(7, device=DEV)).forward(l, i, w)
    c = RtpCombine(2)
    with pytest.raises(ValueError):
        c.forward(torch.zeros(7, 8, device=DEV), None, torch.zeros(4, 8, device=DEV))
    with pytest.raises(ValueError):
        c.forward(torch.zeros(8, 8, device=DEV, dtype=F16), None, torch.zeros(4, 8, device=DEV))
    r.forward(l[:0], i[:0], w[:0])                            # no tokens
    r.backward(l[:0], i[:0], w[:0], l[:0].clone())
    c.forward(torch.zeros(0, 8, device=DEV), None, torch.zeros(0, 8, device=DEV))
