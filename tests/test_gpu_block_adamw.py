"""The AdamW step against its definition in 64 bits.

Tolerances, u = 2^-24: a moment is two products and a sum, with coefficients rounded to fp32 (the square twice): 6 u of the magnitudes added up.
The parameter: 3 u of itself, and of the update what the moments' errors, a root, a quotient and the host's rounded factors
make of it, 24 u and the first moment's error over its denominator.  Whatever is rounded at random is one of the two neighbours,
the one that the random bits (which the tests compute themselves) say, unless the exact value is within the error above
of the border between them."""
import math

import pytest
import torch

import block_reference as ref
from paper_2311_01635_amd import RtpAdamW
from paper_2311_01635_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
LR, WD, STEP, SEED = 3e-3, 0.1, 7, 0x1234ABCD
SIZES = [1, 5, 255, 256, 257, 4096, 4097, 10000]


def _blocks(n):
    return -(-n // ref.BLOCK)


class Problem:
    def __init__(self, sizes, dtype, master, state, seed=0, offset=0, scale=None, grad=1e-2, wd=WD):
        g = self.gen = torch.Generator().manual_seed(seed + sum(sizes))
        rnd = lambda n: torch.randn(n, generator=g)   # noqa: E731
        self.sizes, self.dtype, self.master, self.state, self.scale, self.wd = sizes, dtype, master, state, scale, wd
        N = self.N = sum(_blocks(n) for n in sizes) * ref.BLOCK
        self.p32 = [rnd(n) * 0.02 for n in sizes]
        self.p = [t.to(dtype) for t in self.p32]
        self.g = [rnd(n) * grad * torch.exp(rnd(n)) for n in sizes]
        self.live = torch.zeros(N, dtype=torch.bool)
        self.at, a = [], 0
        for n in sizes:
            self.at.append(a)
            self.live[a:a + n] = True
            a += _blocks(n) * ref.BLOCK
        m, v = rnd(N) * grad * self.live, (rnd(N) * grad).square() * self.live
        if state == "f32":
            self.m, self.v, self.exps = m, v, None
            self.m64, self.v64 = m.double(), v.double()
        else:                                            # any codes are a state; exponents around those of the gradients
            self.m, self.v = (torch.randint(0, 128, (N,), generator=g, dtype=torch.uint8) * self.live for _ in range(2))
            self.m = self.m | (torch.randint(0, 2, (N,), generator=g, dtype=torch.uint8) * 128)
            self.m = torch.where(self.m & 127 > 119, self.m & 0x87, self.m)
            self.v = self.v + 120 * self.live.to(torch.uint8)
            self.v = torch.where(self.v > 247, 3, self.v).to(torch.uint8)
            e = math.frexp(grad)[1] + 126
            self.exps = torch.stack([torch.randint(e - 3, e + 3, (N // ref.BLOCK,), generator=g), torch.randint(2 * e - 131, 2 * e - 127, (N // ref.BLOCK,), generator=g)], 1).to(torch.uint8)
            self.m64, self.v64 = ref.decode(self.m, self.exps[:, 0], ref.TOP_M) * self.live, ref.decode(self.v, self.exps[:, 1], ref.TOP_V) * self.live
        place = lambda t: (torch.cat([torch.zeros(offset, dtype=t.dtype), t, torch.full((8,), 7, dtype=t.dtype)]).to(DEV))   # noqa: E731
        self.whole = [[place(t) for t in ts] for ts in (self.p, self.g, self.p32)]
        view = lambda ts: [w[offset:offset + n] for w, n in zip(ts, sizes)]   # noqa: E731
        self.P, self.G, self.M = (view(ts) for ts in self.whole)
        dev = lambda t: None if t is None else t.to(DEV)   # noqa: E731
        tensors = [dict(param=p, grad=gr, weight_decay=wd if i % 2 == 0 else 0.0, **({"master": mm} if master else {}))
                   for i, (p, gr, mm) in enumerate(zip(self.P, self.G, self.M))]
        self.opt = RtpAdamW(tensors, state, moments=(dev(self.m), dev(self.v), dev(self.exps)))

    def step(self, seed=SEED, **kw):
        gs = None if self.scale is None else torch.tensor([self.scale], device=DEV)
        self.opt.step(LR, STEP, seed=seed, grad_scale=gs, **kw)
        return self

    def flat(self, ts):
        out = torch.zeros(self.N, dtype=torch.float64)
        for a, t in zip(self.at, ts):
            out[a:a + t.numel()] = t.cpu().double()
        return out

    def check(self, seed=SEED):
        live, g = self.live, self.flat(self.g) * (1.0 if self.scale is None else float(torch.tensor(self.scale)))
        wd = self.flat([torch.full((n,), self.wd if i % 2 == 0 else 0.0) for i, n in enumerate(self.sizes)])
        p0 = self.flat(self.p32 if self.master else self.p)
        p, m, v = ref.adamw(p0, g, self.m64, self.v64, LR, wd, STEP)
        dm = 6 * U * (0.9 * self.m64.abs() + 0.1 * g.abs()) + 2.0 ** -148
        dv = 6 * U * (0.999 * self.v64 + 0.001 * g * g) + 2.0 ** -148
        den = torch.sqrt(v / (1 - 0.999 ** STEP)) + 1e-8
        a = LR / (1 - 0.9 ** STEP)
        dp = 3 * U * (p.abs() + p0.abs()) + a / den * (dm + 24 * U * m.abs())
        rm, rv, rp = ref.random_bits(torch.arange(self.N), seed)
        got = self.flat(self.M if self.master else self.P)
        if self.dtype == F32 or self.master:
            assert ((got - p).abs() <= dp)[live].all()
        else:
            e = ref.binade(p)
            bits = 7 if self.dtype == BF16 else 10
            ulp = ref.two((e if self.dtype == BF16 else e.clamp(min=-14)) - bits)
            # (fp16 drops 13 bits, and 13 random ones decide)
            r = rp / 65536.0 if self.dtype == BF16 else torch.where(e >= -14, (rp >> 3) / 8192.0, rp / 65536.0)
            self.between(got, p, ulp, r, dp)
        if self.master:
            for x, y in zip(self.P, self.M):
                assert torch.equal(x, y.to(self.dtype))
        om, ov = (t.cpu().double() for t in self.opt.moments())
        if self.state == "f32":
            assert ((om - m).abs() <= dm)[live].all() and ((ov - v).abs() <= dv)[live].all()
        else:
            E = self.opt.exps.cpu().to(torch.int64)
            for x, want, err, top, k, r in ((om, m, dm, ref.TOP_M, 0, rm), (ov, v, dv, ref.TOP_V, 1, rv)):
                x, want, err = x * live, want * live, err * live
                high, slack = want.abs().view(-1, ref.BLOCK).amax(1), err.view(-1, ref.BLOCK).amax(1)
                assert (E[:, k] >= ref.binade(high - slack) + 127).all() and (E[:, k] <= ref.binade(high + slack) + 127).all()
                last = (E[:, k] - 127 - (top - 1)).repeat_interleave(ref.BLOCK)
                ulp = ref.two(torch.maximum(ref.binade(want), last) - 3)
                self.between(x, want, ulp, r / 65536.0, err, least=k == 1)
            # what is handed out is what the codes stand for
            assert torch.equal(om[live], ref.decode(self.opt.m.cpu(), self.opt.exps[:, 0].cpu(), ref.TOP_M)[live])
            assert torch.equal(ov[live], ref.decode(self.opt.v.cpu(), self.opt.exps[:, 1].cpu(), ref.TOP_V)[live])
        for ts in self.whole[:2] + (self.whole[2:] if self.master else []):
            for w in ts:
                assert (w[-8:] == 7).all()                # what is behind a tensor stays

    def between(self, got, want, ulp, r, err, least=False):
        live = self.live
        place, d = want.abs() / ulp, err / ulp + 2.0 ** -40
        lo, hi = torch.floor(place + r - d), torch.floor(place + r + d)
        if least:
            lo, hi = (torch.where(want > 0, t.clamp_min(1), t) for t in (lo, hi))
        # (err may carry a value over the border of a binade, where the spacing is another one)
        edge = ref.binade(want) != ref.binade((want.abs() + err))
        x = got.abs() / ulp
        ok = ((x >= lo) & (x <= hi)) | (edge & ((got - want).abs() <= 2 * ulp))
        assert ok[live].all()
        assert ((got == 0) | (want == 0) | (torch.sign(got) == torch.sign(want)) | (want.abs() <= err))[live].all()
        assert float(d[live].median()) < 0.01            # (the borders are narrow: the check says something)


@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("dtype,master", [(F32, False), (BF16, True), (BF16, False), (F16, True), (F16, False)])
@pytest.mark.parametrize("scale", [None, 0.37])
def test_step(dtype, master, state, scale):
    Problem(SIZES, dtype, master, state, scale=scale).step().check()


@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("offset", [1, 2, 3, 4])
def test_tensors_off_16_bytes(offset, state):
    Problem([3, 1000, 4099], BF16, True, state, offset=offset).step().check()
    Problem([3, 1000, 4099], F16, False, state, offset=offset).step().check()


@pytest.mark.parametrize("sizes", [[1], [256], [100000], [7] * 300, list(range(1, 90))], ids=lambda s: f"{len(s)}x{s[-1]}")
def test_numbers_of_tensors(sizes):
    Problem(sizes, F32, False, "8bit").step().check()


@pytest.mark.parametrize("grad", [1e-30, 1e-12, 1e6])
def test_sizes_of_gradients(grad):
    """squares that are denormal or vanish in fp32, and large ones"""
    q = Problem([1000, 300], F32, False, "f32", grad=grad).step()
    if grad > 1e-20:
        q.check()
    else:
        assert all(torch.isfinite(t).all() for t in q.P)
    if grad > 1e-20:
        Problem([1000, 300], F32, False, "8bit", grad=grad).step().check()


@pytest.mark.parametrize("state", ["f32", "8bit"])
def test_another_place_of_the_same_tensor_and_repeats(state):
    """the same call on the same state: the same bits; another seed: other ones (where something is rounded at random)"""
    a, b, c = (Problem(SIZES, BF16, False, state).step(seed=s) for s in (1, 1, 2))
    eq = lambda x, y: all(torch.equal(s, t) for s, t in zip(x.P + [x.opt.m, x.opt.v], y.P + [y.opt.m, y.opt.v]))   # noqa: E731
    assert eq(a, b) and not eq(a, c)


def test_fresh_moments_and_many_steps():
    """from zeros, forty steps: fp32 against 64 bits (errors add up step by step: 40 times a step's, relative to what the parameter moved)"""
    g = torch.Generator().manual_seed(0)
    n = 3000
    p0 = torch.randn(n, generator=g)
    p, opt = p0.to(DEV), None
    grad = torch.empty(n, device=DEV)
    opt = RtpAdamW([dict(param=p, grad=grad, weight_decay=0.05)])
    q, m, v = p0.double(), torch.zeros(n).double(), torch.zeros(n).double()
    for t in range(1, 41):
        gr = torch.randn(n, generator=g)
        grad.copy_(gr)
        opt.step(1e-2, t)
        q, m, v = ref.adamw(q, gr.double(), m, v, 1e-2, 0.05, t)
    assert ((p.cpu().double() - q).abs() <= 40 * (6 * U * q.abs() + 1e-2 * 60 * U)).all()
    opt.close()


def test_random_rounding_is_right_on_average():
    """no gradient: a second moment falls by beta2 a step, less than an eightieth of a code's spacing.  500 steps of 65536 equal ones: their
    mean is 0.999^500.  A step's variance is at most f (1 - f) s^2, f s = v / 1000 and s <= v / 8: 1.3e-4 v^2, over 500 steps at most 0.07 of v^2
    in all, so the mean of 65536 is within 0.27 / 256 (relative) at one deviation; six of them"""
    n = 65536
    p, grad = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    v0 = torch.full((n,), 200, dtype=torch.uint8, device=DEV)
    exps = torch.full((n // 256, 2), 127, dtype=torch.uint8, device=DEV)
    opt = RtpAdamW([dict(param=p, grad=grad)], "8bit", moments=(torch.full((n,), 100, dtype=torch.uint8, device=DEV), v0, exps))
    m1, v1 = (float(t.double().mean()) for t in opt.moments())
    steps = 500
    for t in range(1, steps + 1):
        opt.step(0.0, t)
    m2, v2 = (float(t.double().mean()) for t in opt.moments())
    assert abs(v2 / v1 / 0.999 ** steps - 1) < 6 * 0.27 / 256
    # a first moment falls by a tenth: f s = m / 10, s <= m / 8: 1e-3 m^2 a step around a mean that shrinks, 0.06 of it over ten steps;
    # after `steps` it has sunk below every code
    assert abs(m2) <= 1e-6 * m1
    opt.close()


@pytest.mark.parametrize("state", ["f32", "8bit"])
@pytest.mark.parametrize("scale", [math.nan, math.inf, -math.inf])
def test_a_scale_that_is_not_finite_changes_nothing(scale, state):
    q = Problem([1000, 3], BF16, True, state, scale=scale)
    before = [t.clone() for t in (*q.P, *q.M, q.opt.m, q.opt.v)]
    q.step()
    assert all(torch.equal(a, b) for a, b in zip(before, (*q.P, *q.M, q.opt.m, q.opt.v)))


def test_gradients_that_are_not_finite_stay_in_their_block():
    q = Problem([1000], F32, False, "8bit")
    q.G[0][300] = math.nan
    q.G[0][600] = math.inf
    q.step()
    m, v = q.opt.moments()
    bad = torch.zeros(q.N, dtype=torch.bool, device=DEV)
    bad[256:768] = True
    assert torch.isnan(m[bad]).all() and torch.isnan(v[bad]).all() and torch.isfinite(m[~bad]).all() and torch.isfinite(v[~bad]).all()
    fine = torch.ones(1000, dtype=torch.bool, device=DEV)
    fine[[300, 600]] = False
    assert torch.isfinite(q.P[0][fine]).all() and not torch.isfinite(q.P[0][300])


def test_empty_blocks_stay_zero():
    p, g = torch.zeros(1000, device=DEV, dtype=BF16), torch.zeros(1000, device=DEV)
    for state in ("f32", "8bit"):
        opt = RtpAdamW([dict(param=p, grad=g, weight_decay=0.1)], state)
        for t in range(1, 4):
            opt.step(1e-3, t)
        assert (p == 0).all() and (opt.m == 0).all() and (opt.v == 0).all()


def test_scalars_from_the_device():
    a, b = Problem(SIZES, BF16, False, "8bit"), Problem(SIZES, BF16, False, "8bit")
    sc = RtpAdamW.scalars_of(LR, STEP, seed=SEED).to(DEV)
    a.step()
    b.opt.step(None, None, scalars=sc)
    assert all(torch.equal(x, y) for x, y in zip(a.P + [a.opt.m, a.opt.v], b.P + [b.opt.m, b.opt.v]))
    with pytest.raises(ValueError):
        b.opt.step(None, None, scalars=sc[:40])


def test_moments_types():
    q = Problem([500], F32, False, "8bit")
    m, v = q.opt.moments(F32)
    bm, bv = q.opt.moments()
    assert torch.equal(m, bm.float()) and torch.equal(v, bv.float()) and torch.equal(m.cpu().double()[q.live], q.m64[q.live])
    q = Problem([500], F32, False, "f32")
    assert torch.equal(q.opt.moments()[0], q.opt.m) and torch.equal(q.opt.moments(BF16)[1], q.opt.v.bfloat16())
    with pytest.raises(B.RtpError):
        q.opt.moments(F16)


def test_refusals_on_the_device():
    t = lambda n, dt=F32: torch.zeros(n, dtype=dt, device=DEV)   # noqa: E731
    p, g = t(100, BF16), t(100)
    for bad in (dict(param=p, grad=g.half()), dict(param=p, grad=g[:99]), dict(param=t(200, BF16)[::2], grad=g), dict(param=p, grad=g.cpu()),
                dict(param=p, grad=g, master=t(99)), dict(param=t(100, torch.float64), grad=g), dict(param=t(0), grad=t(0))):
        with pytest.raises(ValueError):
            RtpAdamW([bad])
    for bad in ([dict(param=p, grad=g)] * 2, [dict(param=g, grad=g)], [dict(param=t(100), grad=g, master=t(100))], [dict(param=p, grad=g, weight_decay=math.nan)]):
        with pytest.raises(B.RtpError):
            RtpAdamW(bad)
    with pytest.raises(ValueError):
        RtpAdamW([dict(param=p, grad=g)], "8bit", moments=(t(256, torch.uint8), t(256, torch.uint8), t(2, torch.uint8)))
    opt = RtpAdamW([dict(param=p, grad=g)])
    for kw in (dict(lr=math.nan, step=1), dict(lr=1e-3, step=0), dict(lr=1e-3, step=1, eps=0.0), dict(lr=1e-3, step=1, betas=(1.0, 0.9))):
        with pytest.raises(B.RtpError):
            opt.step(**kw)
    for scale in (torch.ones(1), torch.ones(2, device=DEV), torch.ones(1, device=DEV, dtype=torch.float64), 0.5):
        with pytest.raises(ValueError):
            opt.step(1e-3, 1, grad_scale=scale)
