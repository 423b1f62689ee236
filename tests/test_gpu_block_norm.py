"""Norms, gate and residual between units against their definitions in 64 bits.

Tolerances, u = 2^-24.  Forward: a row's deviation is a sum of D squares, each lane adding at most D / 64 of them (a row of more than 2048
has more lanes): (D / 64 + 16) u of itself; a mean's error counts as often as the mean is larger than the deviation.  So a
normalised value is off by at most c u (|n| + |mu| rs), c = D / 64 + 24, and everything after it rounds a few times more.  h is
compared with the norm of r as stored.  Backward: the same c on every term that is added up, means taken over magnitudes.  Sums over
rows: T u of the sum of magnitudes more.  16-bit outputs: half a step of their type on top."""
import math

import pytest
import torch

import block_reference as ref
from paper_2311_01635_amd import RtpNorm

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
EPS = 1e-5
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(F32, F32), (F32, BF16), (F32, F16), (BF16, BF16), (F16, F16)]
SHAPES = [(1, 1), (2, 3), (3, 64), (17, 72), (5, 511), (130, 768), (4, 1000), (33, 1024), (2, 2048), (6, 2056), (3, 4096), (2, 5003), (3, 8192), (2, 12296), (2, 16384), (1, 40000)]
PARTS = [  # join, post, pre, gate, affine
    (True, True, True, "channel", True), (True, True, True, "element", True), (True, True, True, "none", False), (True, False, True, "none", True),
    (True, False, True, "channel", True), (True, False, True, "element", False), (True, True, False, "channel", True), (True, False, False, "element", True),
    (False, False, True, "none", True), (False, False, True, "none", False), (True, True, False, "none", True), (True, False, False, "none", False)]


def _half(dt):
    return torch.finfo(dt).eps / 2


def _tiny(dt):
    return 2.0 ** -25 if dt == F16 else 0.0


class Problem:
    """inputs (on the CPU, in their types), the object, and what 64 bits say"""

    def __init__(self, T, D, kind, types, parts, seed=0, mean=0.3, bias=True, alpha=0.75, beta=-1.25):
        self.T, self.D, self.kind, (self.S, self.B) = T, D, kind, types
        self.join, self.post, self.pre, self.gate_kind, affine = parts
        self.alpha, self.beta = (alpha, beta) if self.join else (1.0, 1.0)
        g = self.gen = torch.Generator().manual_seed(seed + T * 31 + D)
        rnd = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
        self.x, self.y = (rnd(T, D) * 2 + mean).to(self.S), (rnd(T, D) + mean).to(self.B)
        vec = lambda shift: rnd(D) * 0.2 + shift        # noqa: E731
        self.p = {}
        if affine:
            if self.post:
                self.p["w_post"] = vec(1.0)
                if bias:
                    self.p["b_post"] = vec(0.0)
            if self.pre:
                self.p["w_pre"] = vec(1.0)
                if bias:
                    self.p["b_pre"] = vec(0.0)
        if self.gate_kind == "channel":
            self.p["gate"] = vec(0.5)
        self.gate = (rnd(T, D) * 0.3 + 0.5).to(self.B) if self.gate_kind == "element" else None
        self.norm = RtpNorm(D, kind=kind, eps=EPS, join=self.join, post=self.post, pre=self.pre, res_scale=self.alpha, out_scale=self.beta,
                            stream_dtype=self.S, dtype=self.B, **{k: v.to(DEV) for k, v in self.p.items()})
        self.c = (D / 64 + 24) * U

    def d(self, t):
        return None if t is None else t.double()

    def gate64(self):
        return self.d(self.p.get("gate")) if self.gate is None else self.d(self.gate)

    def forward(self, x=None, y=None):
        self.xd, self.yd, self.gd = (None if t is None else t.to(DEV) for t in (self.x if x is None else x, self.y if y is None else y, self.gate))
        self.r = torch.full((self.T, self.D), math.nan, dtype=self.S, device=DEV) if self.join else None
        self.h = torch.full((self.T, self.D), math.nan, dtype=self.B, device=DEV) if self.pre else None
        self.stats = torch.full((self.T, 4), math.nan, device=DEV)
        self.norm.forward(self.xd, self.yd if self.join else None, self.r, self.h, self.stats, gate=self.gd)
        return self

    def size(self, v, w, b):
        """bound of |N(v)|'s terms"""
        mu, rs = ref.stats(v, self.kind, EPS)
        s = ((v - mu[:, None]).abs() + 2 * mu.abs()[:, None]) * rs[:, None]
        return s * (1.0 if w is None else w.abs()) + (0.0 if b is None else b.abs())

    def check_forward(self):
        x, y, p = self.x.double(), self.y.double(), {k: v.double() for k, v in self.p.items()}
        stream = x
        if self.join:
            g = self.gate64()
            want = ref.join(x, y, self.kind, EPS, self.post, self.alpha, self.beta, p.get("w_post"), p.get("b_post"), g)
            branch = (self.size(y, p.get("w_post"), p.get("b_post")) if self.post else y.abs()) * (1.0 if g is None else g.abs())
            tol = _half(self.S) * want.abs() * 1.01 + self.c * (abs(self.alpha) * x.abs() + abs(self.beta) * branch) + _tiny(self.S)
            assert ((self.r.cpu().double() - want).abs() <= tol).all()
            stream = self.r.cpu().double()
        if self.pre:
            want = ref.norm(stream, self.kind, EPS, p.get("w_pre"), p.get("b_pre"))
            tol = _half(self.B) * want.abs() * 1.01 + self.c * self.size(stream, p.get("w_pre"), p.get("b_pre")) + _tiny(self.B)
            assert ((self.h.cpu().double() - want).abs() <= tol).all()
        st = self.stats.cpu().double()
        for on, v, at in ((self.post, y, 0), (self.pre, stream, 2)):
            if on:
                mu, rs = ref.stats(v, self.kind, EPS)
                assert ((st[:, at] - mu).abs() <= self.c * v.abs().mean(1)).all()
                assert ((st[:, at + 1] - rs).abs() <= self.c * rs * (1 + mu.abs() * rs)).all()
            else:
                assert torch.isnan(st[:, at:at + 2]).all()

    def backward(self, dr=True, **kw):
        rnd = lambda: torch.randn(self.T, self.D, generator=self.gen)   # noqa: E731
        self.dr = rnd().to(self.S) if dr or not self.pre else None
        self.dh = rnd().to(self.B) if self.pre else None
        new = lambda dt: torch.full((self.T, self.D), math.nan, dtype=dt, device=DEV)   # noqa: E731
        self.dx, self.dy = new(self.S), new(self.B) if self.join else None
        self.dgate = new(self.B) if self.gate is not None else None
        to = lambda t: None if t is None else t.to(DEV)                 # noqa: E731
        self.grads = self.norm.backward(self.r if self.join else self.xd, self.yd, to(self.dr), to(self.dh), self.dx, self.dy, self.stats, gate=self.gd,
                                        dgate=self.dgate, **kw)
        return self

    def expected(self):
        """gradients by autograd in 64 bits, at the stored r: {name: (value, magnitude of what is added up)}"""
        p = {k: v.double().requires_grad_() for k, v in self.p.items()}
        x, y = self.x.double().requires_grad_(), self.y.double().requires_grad_()
        e = None if self.gate is None else self.gate.double().requires_grad_()
        dR = torch.zeros(self.T, self.D, dtype=torch.float64) if self.dr is None else self.dr.double()
        mag = dR.abs()
        out, back = {}, lambda n, rs, dn: rs * (dn.abs() + dn.abs().mean(1, keepdim=True) + n * (dn.abs() * n).mean(1, keepdim=True))   # noqa: E731
        if self.pre:
            s = (self.r.cpu() if self.join else self.x).double().requires_grad_()
            h = ref.norm(s, self.kind, EPS, p.get("w_pre"), p.get("b_pre"))
            (h * self.dh.double()).sum().backward()
            n, dh = self.size(s.detach(), None, None), self.dh.double()
            dR = dR + s.grad
            mag = mag + back(n, ref.stats(s.detach(), self.kind, EPS)[1][:, None], dh * (self.p["w_pre"].double() if "w_pre" in p else 1.0))
            for name, m in (("w_pre", dh.abs() * n), ("b_pre", dh.abs())):
                if name in p:
                    out[name] = (p[name].grad, m.sum(0))
        if not self.join:
            out["dx"] = (dR, mag)
            return out
        g = e if e is not None else p.get("gate")
        r = ref.join(x, y, self.kind, EPS, self.post, self.alpha, self.beta, p.get("w_post"), p.get("b_post"), g)
        (r * dR).sum().backward()
        out["dx"] = (x.grad, abs(self.alpha) * mag)
        b = abs(self.beta) * mag
        o = self.size(y.detach(), p["w_post"].detach() if "w_post" in p else None, p["b_post"].detach() if "b_post" in p else None) if self.post else y.detach().abs()
        if e is not None:
            out["dgate"] = (e.grad, b * o)
        elif "gate" in p:
            out["gate"] = (p["gate"].grad, (b * o).sum(0))
        b = b * (1.0 if g is None else g.detach().abs())
        if self.post:
            n = self.size(y.detach(), None, None)
            for name, m in (("w_post", b * n), ("b_post", b)):
                if name in p:
                    out[name] = (p[name].grad, m.sum(0))
            b = back(n, ref.stats(y.detach(), self.kind, EPS)[1][:, None], b * (p["w_post"].detach().abs() if "w_post" in p else 1.0))
        out["dy"] = (y.grad, b)
        return out

    def check_backward(self, start=None):
        want = self.expected()
        got = {"dx": self.dx, "dy": self.dy, "dgate": self.dgate, **self.grads}
        assert {k for k, v in got.items() if v is not None} == set(want)
        for name, (v, m) in want.items():
            x = got[name].cpu().double()
            half = _half(got[name].dtype) if name in ("dx", "dy", "dgate") else U
            v = v if start is None or name in ("dx", "dy", "dgate") else v + start
            rows = self.T if name not in ("dx", "dy", "dgate") else 0
            # (three sums over the row one after the other: 3 c)
            tol = half * v.abs() * 1.01 + (3 * self.c + rows * U) * m + _tiny(got[name].dtype)
            assert ((x - v).abs() <= tol).all(), (name, float(((x - v).abs() / tol.clamp_min(1e-300)).max()))


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("types", [TYPES[1], TYPES[3]], ids=str)
def test_shapes(shape, types, kind):
    for parts in (PARTS[0], PARTS[1], PARTS[3]):
        q = Problem(*shape, kind, types, parts).forward()
        q.check_forward()
        q.backward().check_backward()


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("parts", PARTS, ids=str)
def test_parts_and_types(parts, types, kind):
    for (T, D), bias in (((41, 264), True), ((7, 1203), False)):
        q = Problem(T, D, kind, types, parts, bias=bias).forward()
        q.check_forward()
        q.backward(dr=T == 41).check_backward()


@pytest.mark.parametrize("T", [1, 255, 1025, 5000])
def test_many_rows_and_adding_up(T):
    """sums over more rows than there are partial sums; a second pass adds to the first, a third overwrites; bit for bit again"""
    q = Problem(T, 136, "layer", (BF16, BF16), PARTS[0]).forward()
    for t in q.norm.grads.values():
        t.fill_(2.5)
    q.backward().check_backward(start=2.5)
    q.norm.zero_grads()
    q.backward().check_backward()
    q.backward(accumulate=False).check_backward()
    first = {k: v.clone() for k, v in q.grads.items()}
    to = lambda t: t.to(DEV)   # noqa: E731
    q.norm.backward(q.r, q.yd, to(q.dr), to(q.dh), q.dx, q.dy, q.stats, accumulate=False)
    assert all(torch.equal(first[k], q.grads[k]) for k in first)


def test_values_far_from_zero_and_rows_of_one_value():
    """a mean a thousand deviations away; rows without deviation; rows of zeros"""
    q = Problem(9, 512, "layer", (F32, F32), PARTS[0], mean=1000.0).forward()
    q.check_forward()
    q.backward().check_backward()
    for kind in ("rms", "layer"):
        q = Problem(4, 300, kind, (F32, F32), PARTS[2])
        q.x[0], q.y[0], q.x[1], q.y[1] = 0.0, 0.0, 7.0, -3.0
        q.forward().check_forward()
        q.backward()
        assert all(torch.isfinite(t).all() for t in (q.r, q.h, q.dx, q.dy))


def test_large_and_infinite_rows_stay_in_their_row():
    q = Problem(6, 640, "rms", (F32, BF16), PARTS[0])
    q.y[2, 5] = math.inf
    q.y[4, 7] = math.nan
    q.forward()
    ok = [0, 1, 3, 5]
    assert torch.isfinite(q.r[ok]).all() and torch.isfinite(q.h[ok]).all()
    assert torch.isnan(q.r[2]).any() and torch.isnan(q.r[4]).all()


@pytest.mark.parametrize("types", [(BF16, BF16), (F32, BF16)], ids=str)
@pytest.mark.parametrize("off,pad,D", [(0, 8, 264), (1, 2, 264), (8, 5, 1200), (3, 0, 77), (4, 4, 4100)])
def test_strides_and_in_place(off, pad, D, types):
    """columns that start off 16 bytes, rows apart, r in the place of x, dx in that of dr: the values are those of whole tensors, and what
    lies between the rows and behind them stays"""
    T = 11
    q = Problem(T, D, "layer", types, PARTS[1]).forward()
    q.check_forward()

    def view(t):
        w = torch.full((T + 1, D + off + pad), 9.0, dtype=t.dtype, device=DEV)
        w[:T, off:off + D].copy_(t)
        return w, w[:T, off:off + D]
    x, y, h, gate = view(q.x), view(q.y), view(q.h), view(q.gate)
    stats = torch.empty(T, 4, device=DEV)
    q.norm.forward(x[1], y[1], x[1], h[1], stats, gate=gate[1])
    q2 = Problem(T, D, "layer", types, PARTS[1])
    q2.r, q2.h, q2.stats = x[1].clone(), h[1].clone(), stats
    q2.check_forward()
    q.backward().check_backward()
    # ... from the first pass's r and stats, so that only the strides differ
    r, dr, dh, dy, dgate = view(q.r), view(q.dr), view(q.dh), view(q.dy), view(q.dgate)
    q.norm.zero_grads()
    q.norm.backward(r[1], y[1], dr[1], dh[1], dr[1], dy[1], q.stats, gate=gate[1], dgate=dgate[1])
    q.dx, q.dy, q.dgate = dr[1].clone(), dy[1].clone(), dgate[1].clone()
    q.check_backward()
    for w, v in (x, h, dr, dy, dgate):
        v.fill_(9.0)
        assert (w == 9.0).all()


def test_gradient_by_differences():
    """along a direction in every input at once: what 64 bits give for the loss a small step to either side, against the kernel's gradient"""
    for kind in ("rms", "layer"):
        q = Problem(6, 96, kind, (F32, F32), PARTS[0]).forward().backward()
        g = torch.Generator().manual_seed(4)
        d = {k: torch.randn(v.shape, generator=g).double() for k, v in (("x", q.x), ("y", q.y), *q.p.items())}

        def loss(s):
            p = {k: v.double() + s * d[k] for k, v in q.p.items()}
            r = ref.join(q.x.double() + s * d["x"], q.y.double() + s * d["y"], kind, EPS, True, q.alpha, q.beta, p["w_post"], p.get("b_post"), p["gate"])
            return float((r * q.dr.double()).sum() + (ref.norm(r, kind, EPS, p["w_pre"], p.get("b_pre")) * q.dh.double()).sum())
        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        got = {"x": q.dx, "y": q.dy, **q.grads}
        along = sum(float((got[k].cpu().double() * d[k]).sum()) for k in d)
        want = q.expected()
        mags = sum(float((want["d" + k if k in "xy" else k][1] * d[k].abs()).sum()) for k in d)
        # the kernel's errors, r's own rounding (u, through a second derivative of order 1), and the differences' truncation
        assert abs(along - slope) <= (4 * q.c + 10 * U + 1e-7) * mags


@pytest.mark.parametrize("D", [96, 1000, 17000])
def test_any_of_the_parameter_gradients_alone(D):
    """through the C ABI: each gradient by itself, and all but it, are those of the call that asks for all; the others stay as they were"""
    import ctypes as C

    from paper_2311_01635_amd import binding as B
    q = Problem(300 if D < 2000 else 5, D, "layer", (BF16, BF16), PARTS[0]).forward().backward()
    full = {k: v.clone() for k, v in q.grads.items()}
    keep = [t.to(DEV) for t in (q.dr, q.dh)]
    names = {"w_post": "dw_post_dev", "b_post": "db_post_dev", "w_pre": "dw_pre_dev", "b_pre": "db_pre_dev", "gate": "dgate_dev"}
    d = B.rtp_norm_desc.from_buffer_copy(q.norm.desc)
    d.T = q.T
    ws = torch.empty(B.lib.rtp_norm_ws_bytes(C.byref(d)), dtype=torch.uint8, device=DEV)
    for name in names:
        for wanted in ([name], [n for n in names if n != name]):
            g = B.rtp_norm_grads()
            g.r_dev, g.y_dev, g.dr_dev, g.dh_dev, g.stats_dev = (t.data_ptr() for t in (q.r, q.yd, *keep, q.stats))
            g.dx_dev, g.dy_dev, g.ws_dev, g.ws_bytes = q.dx.data_ptr(), q.dy.data_ptr(), ws.data_ptr(), ws.numel()
            got = {n: torch.full((D,), 4.0, device=DEV) for n in names}
            for n in wanted:
                setattr(g, names[n], got[n].data_ptr())
            B.check(B.lib.rtp_norm_bwd(C.byref(d), C.byref(g), torch.cuda.current_stream().cuda_stream))
            assert all(torch.equal(got[n], full[n]) if n in wanted else (got[n] == 4.0).all() for n in names), wanted


def test_batches_of_changing_size():
    """one object, one batch after another of another number of rows: each call has the workspace of its own"""
    for T in (700, 3, 5000, 1, 700):
        q = Problem(T, 96, "rms", (BF16, BF16), PARTS[0])
        if T == 700:
            first = q
        q.norm, q.p = first.norm, first.p
        q.forward().backward(accumulate=False).check_backward()


def test_an_element_gate_without_its_gradient():
    q = Problem(9, 264, "rms", (BF16, BF16), PARTS[1]).forward().backward()
    dx, dy = torch.empty_like(q.dx), torch.empty_like(q.dy)
    q.norm.backward(q.r, q.yd, q.dr.to(DEV), q.dh.to(DEV), dx, dy, q.stats, gate=q.gd)
    assert torch.equal(dx, q.dx) and torch.equal(dy, q.dy)


def test_refusals_on_the_device():
    n = RtpNorm(16, post=True, w_pre=torch.ones(16, device=DEV))
    t = lambda *s, dt=BF16: torch.zeros(*s, dtype=dt, device=DEV)   # noqa: E731
    ok = [t(4, 16), t(4, 16), t(4, 16), t(4, 16), t(4, 4, dt=F32)]
    n.forward(*ok)
    for i, bad in ((0, t(4, 17)), (0, t(4, 16, dt=F32)), (1, t(3, 16)), (1, None), (2, None), (3, t(4, 32)[:, ::2]), (4, t(4, 3, dt=F32)), (4, None), (2, t(1, 16).expand(4, 16))):
        a = list(ok)
        a[i] = bad
        with pytest.raises(ValueError):
            n.forward(*a)
    from paper_2311_01635_amd import binding as B
    with pytest.raises(B.RtpError):
        n.forward(ok[0], ok[1], ok[1], ok[3], ok[4])
    with pytest.raises(ValueError):
        RtpNorm(16, gate=torch.ones(16, device=DEV)).forward(*ok, gate=t(4, 16))
    with pytest.raises(ValueError):
        n.backward(ok[0], ok[1], None, ok[2], t(4, 16), t(4, 16), ok[4], dgate=t(4, 16))
    n.forward(*[a[:0] for a in ok])                             # no tokens
    n.grads["w_pre"].fill_(3.0)
    empty = [a[:0] for a in (ok[0], ok[1], t(4, 16), ok[2], t(4, 16), t(4, 16), ok[4])]
    n.backward(*empty)
    assert (n.grads["w_pre"] == 3.0).all()
    n.backward(*empty, accumulate=False)
    assert (n.grads["w_pre"] == 0.0).all()
