"""The operators around a unit together, as a training step uses them: norm, router, experts, combination, residual, back, AdamW; on
other streams and in graphs."""
import math

import numpy as np
import pytest
import torch

import block_reference as ref
import rtp_workloads as wl
from paper_2311_01635_amd import RtpAdamW, RtpCombine, RtpNorm, RtpRouter
from paper_2311_01635_amd import binding as B
from paper_2311_01635_amd.layers import RtpLinear, RtpMlp, RtpMoe

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32
BAR = 2e-2   # the framework's bar for 16-bit units: max-norm relative error


def _dev(a, dt):
    return (torch.from_numpy(np.ascontiguousarray(a)) if isinstance(a, np.ndarray) else a).to(DEV, dt)


def _new(*s, dt=BF):
    return torch.full(s, math.nan, dtype=dt, device=DEV)


def _err(got, want):
    got, want = got.detach().cpu().double(), want.detach().double()
    return float((got - want).abs().max() / want.abs().max())


def _expert(x, ex, gated):
    if gated:
        return (torch.nn.functional.silu(x @ ex[0].t()) * (x @ ex[1].t())) @ ex[2].t()
    return torch.nn.functional.gelu(x @ ex[0].t()) @ ex[1].t()


@pytest.mark.parametrize("gated,k,n", [(True, 2, 4), (False, 3, 4), (False, 1, 3)])
def test_block_with_experts(gated, k, n):
    """x -> norm -> router -> top-k experts -> weighted -> norm, channel gate, residual -> norm of the next unit, and all gradients"""
    T, I, O = 96, 128, 192
    inp = wl.make_moe_inputs(T, I, O, I, n, gated=gated, seed=1)
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g)   # noqa: E731
    x, Wr = rnd(T, I).to(BF), (rnd(n, I) * 0.2).to(BF)
    w1, w2, w3, gate = (1 + 0.1 * rnd(I) for _ in range(4))
    dr, dh = rnd(T, I).to(BF), rnd(T, I).to(BF)
    moe = RtpMoe([tuple(_dev(m, BF) for m in ex) for ex in inp["experts"]], T, 1, B.RTP_ACT_SWIGLU if gated else B.RTP_ACT_GELU_ERF, top_k=k)
    pre = RtpNorm(I, join=False, w_pre=w1.to(DEV))
    post = RtpNorm(I, post=True, w_post=w2.to(DEV), gate=gate.to(DEV), w_pre=w3.to(DEV), out_scale=0.5)
    router = RtpRouter(n, k)
    xd = x.to(DEV)
    h, st1, logits, ids, wt = _new(T, I), _new(T, 4, dt=F32), _new(T, n, dt=F32), torch.empty(T, k, dtype=torch.int32, device=DEV), _new(T, k, dt=F32)
    y, r, h2, st2 = _new(T, I), _new(T, I), _new(T, I), _new(T, 4, dt=F32)
    pre.forward(xd, None, None, h, st1)
    torch.matmul(h.float(), Wr.to(DEV).float().t(), out=logits)
    router.forward(logits, ids, wt)
    moe.forward(h, ids, y, wt)
    post.forward(xd, y, r, h2, st2)
    # back
    dx, dy, dwt, dl, dhx, dx0 = _new(T, I), _new(T, I), _new(T, k, dt=F32), _new(T, n, dt=F32), _new(T, I), _new(T, I)
    post.backward(r, y, dr.to(DEV), dh.to(DEV), dx, dy, st2)
    moe.backward(dy, dhx, wt, dwt)
    router.backward(logits, ids, dwt, dl)
    dhx = (dhx.float() + dl @ Wr.to(DEV).float()).to(BF)
    pre.backward(xd, None, dx, dhx, dx0, None, st1)
    moe.sync()
    # the same in 64 bits, with the kernel's choice of experts
    leaf = lambda t: torch.as_tensor(t).double().requires_grad_()   # noqa: E731
    X, R, a1, a2, a3, ga = leaf(x), leaf(Wr), leaf(w1), leaf(w2), leaf(w3), leaf(gate)
    exs = [tuple(leaf(m) for m in ex) for ex in inp["experts"]]
    H = ref.norm(X, "rms", 1e-5, a1)
    W = ref.route_weights(H @ R.t(), ids.cpu(), "softmax", True, 1.0)
    outs = torch.stack([_expert(H, ex, gated) for ex in exs], 1)                          # [T, n, I]
    Y = (W[:, :, None] * outs.gather(1, ids.cpu().long()[:, :, None].expand(T, k, I))).sum(1)
    Rr = ref.join(X, Y, "rms", 1e-5, True, 1.0, 0.5, a2, None, ga)
    H2 = ref.norm(Rr, "rms", 1e-5, a3)
    ((Rr * dr.double()).sum() + (H2 * dh.double()).sum()).backward()
    for name, got, want in (("h", h, H), ("weights", wt, W), ("y", y, Y), ("r", r, Rr), ("h2", h2, H2), ("dx", dx0, X.grad), ("w1", pre.grads["w_pre"], a1.grad),
                            ("w2", post.grads["w_post"], a2.grad), ("w3", post.grads["w_pre"], a3.grad), ("gate", post.grads["gate"], ga.grad)):
        assert _err(got, want) <= BAR, name
    if k > 1:
        # (through bf16 rows: the dot products behind it are of 128 rounded values, a few of which nearly cancel)
        assert _err(dl.t() @ h.float(), R.grad) <= 2 * BAR
    _, grads = moe.gathered()
    for e in range(n):
        for got, want in zip(grads[e], exs[e]):
            if float(want.grad.abs().max()) > 0:
                assert _err(got, want.grad) <= BAR, e
            else:                                       # an expert that no token went to
                assert (got == 0).all()
    moe.close()


def test_moe_without_weights_is_what_it_was():
    """top_k = 1 and no weights: rtp_moe_fwd / rtp_moe_bwd themselves; with weights of 1 the same numbers"""
    T, I, O, n = 64, 128, 128, 4
    inp = wl.make_moe_inputs(T, I, O, I, n, seed=3)
    res = []
    for weights in (None, torch.ones(T, 1, device=DEV)):
        moe = RtpMoe([tuple(_dev(m, BF) for m in ex) for ex in inp["experts"]], T, 0, B.RTP_ACT_GELU_ERF)
        X, route, dY = _dev(inp["X"], BF), _dev(inp["route"], torch.int32), _dev(inp["dY"], BF)
        Y, dX = _new(T, I), _new(T, I)
        moe.forward(X, route if weights is None else route.view(T, 1), Y, weights)
        moe.backward(dY, dX, weights)
        moe.sync()
        res.append((Y, dX))
        moe.close()
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])


def test_weighted_moe_calls_from_several_streams():
    """calls that nothing but the layer itself orders (each on a stream of its own, the compute stream held back): the slots' rows of one
    are not overwritten by the next"""
    T, I, O, n, k = 64, 128, 128, 4, 2
    inp = wl.make_moe_inputs(T, I, O, I, n, seed=3)
    moe = RtpMoe([tuple(_dev(m, BF) for m in ex) for ex in inp["experts"]], T, 0, B.RTP_ACT_GELU_ERF, top_k=k)
    g = torch.Generator(device=DEV).manual_seed(1)
    calls = []
    for _ in range(4):
        X, dY = (torch.randn(T, I, generator=g, device=DEV).to(BF) for _ in range(2))
        ids = torch.stack([torch.randperm(n, generator=g, device=DEV)[:k] for _ in range(T)]).int()
        calls.append((X, dY, ids, torch.rand(T, k, generator=g, device=DEV), [_new(T, I), _new(T, I), _new(T, k, dt=F32)]))

    def run(c):
        X, dY, ids, w, (Y, dX, dw) = c
        moe.forward(X, ids, Y, w)
        moe.backward(dY, dX, w, dw)
    want = []
    for c in calls:
        run(c)
        moe.sync()
        want.append([t.clone() for t in c[4]])
        for t in c[4]:
            t.fill_(math.nan)
    scratch = torch.zeros(16, dtype=torch.uint8, device=DEV)
    B.check(B.lib.rtp_ring_set_test_delay_compute(moe.ring_handle(), scratch.data_ptr(), 100))
    torch.cuda.synchronize()
    for c in calls:
        with torch.cuda.stream(torch.cuda.Stream()):
            run(c)
    torch.cuda.synchronize()
    for c, w in zip(calls, want):
        assert _same(c[4], w)
    moe.close()


def test_moe_refuses_a_route_of_another_shape():
    T, I, n = 64, 128, 2
    inp = wl.make_moe_inputs(T, I, 128, I, n, seed=3)
    moe = RtpMoe([tuple(_dev(m, BF) for m in ex) for ex in inp["experts"]], T, 0, B.RTP_ACT_GELU_ERF, top_k=2)
    X, Y = _dev(inp["X"], BF), _new(T, I)
    for route in (torch.zeros(T, dtype=torch.int32, device=DEV), torch.zeros(T, 2, dtype=torch.int64, device=DEV), torch.zeros(T, 3, dtype=torch.int32, device=DEV)):
        with pytest.raises(ValueError):
            moe.forward(X, route, Y)
    moe.close()


@pytest.mark.parametrize("state,master", [("f32", True), ("f32", False), ("8bit", False)])
def test_optimizer_over_ring_stores(state, master):
    """three training steps of two layers and a norm's weight: the stores' weights follow the definition, gradients begin at zero each step"""
    T, I, O, n = 64, 96, 160, 4
    g = torch.Generator().manual_seed(5)
    W1, W2 = torch.randn(O, I, generator=g) * 0.05, torch.randn(I, O, generator=g) * 0.05
    Wl = torch.randn(O, I, generator=g) * 0.05
    mlp = RtpMlp([W1, W2], T, n, 1, B.RTP_ACT_GELU_ERF)
    lin = RtpLinear(Wl, T, n, 2)
    nw, ng = torch.ones(I, device=DEV), torch.zeros(I, device=DEV)
    opt = RtpAdamW.for_layers([mlp, lin], state, master=master, weight_decay=0.1, more=[dict(param=nw, grad=ng)])
    X, dY, dYl = (torch.randn(T, w, generator=g).to(BF).to(DEV) for w in (I, I, O))
    Y, dX, Yl = _new(T, I), _new(T, I), _new(T, O)
    lr, step64 = 1e-3, {}
    for t in range(1, 4):
        mlp.forward(X, Y)
        mlp.backward(X, dY, dX)
        lin.forward(X, Yl)
        lin.backward(X, dYl, dX)
        ng.copy_(X.float().mean(0))
        before = [w.double().cpu() for w in (*mlp.gathered()[0], lin.gathered()[0], nw)]
        grads = [x.double().cpu() for x in (*mlp.gathered()[1], lin.gathered()[1], ng)]
        assert all(float(x.abs().max()) > 0 for x in grads)
        opt.step(lr, t)
        after = [w.double().cpu() for w in (*mlp.gathered()[0], lin.gathered()[0], nw)]
        cleared = (*mlp.gathered()[1], lin.gathered()[1])
        assert all((x == 0).all() for x in cleared)
        for i, (b, a, gr) in enumerate(zip(before, after, grads)):
            m, v = step64.get(i, (torch.zeros_like(b), torch.zeros_like(b)))
            p, m, v = ref.adamw(b, gr, m, v, lr, 0.1 if i < 3 else 0.0, t)
            step64[i] = (m, v)
            # half a step of bf16 is 2^-8 of the value.  Without a copy the step begins at b itself and its result p goes to either
            # neighbour: a step, 2 half |p|.  With one, b is the copy to half |b| and a the new copy to half |p|.  8-bit
            # moments are off by an eighth at most each, so that an update of about lr is by 0.4 of it
            half = 2.0 ** -8
            tol = (half * (2 * p.abs() + b.abs()) * 1.01 if i < 3 else 0) + (0.4 * lr * t if state == "8bit" else 0) + 1e-5 * lr + 2.0 ** -23 * p.abs()
            assert ((a - p).abs() <= tol).all(), (t, i)
            assert float((a - b).abs().max()) > 0
    mlp.close()
    lin.close()
    opt.close()


class Chain:
    """norm -> router -> combination -> norm, back, and a step of the norm's parameters: everything that may be captured"""

    def __init__(self, T=70, D=264, E=24, k=3, seed=0):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)   # noqa: E731
        self.T, self.D, self.k = T, D, k
        self.x, self.y, self.logits, self.yk = rnd(T, D), rnd(T, D).to(BF), rnd(T, E), rnd(T * k, D).to(BF)
        self.dr, self.dh = rnd(T, D), rnd(T, D).to(BF)
        self.norm = RtpNorm(D, kind="layer", post=True, w_post=rnd(D), b_post=rnd(D), gate=rnd(D), w_pre=rnd(D), b_pre=rnd(D), stream_dtype=F32)
        self.router, self.combine = RtpRouter(E, k, score="sigmoid", groups=4, kept_groups=2, group_top=2, bias=0.1 * rnd(E)), RtpCombine(k)
        self.opt = RtpAdamW([dict(param=p, grad=self.norm.grads[n], weight_decay=0.1) for n, p in self.norm.params.items()], "8bit")
        self.scalars = RtpAdamW.scalars_of(1e-2, 1).to(DEV)
        self.ids, self.w, self.yc = torch.empty(T, k, dtype=torch.int32, device=DEV), _new(T, k, dt=F32), _new(T, D)
        self.r, self.h, self.stats = _new(T, D, dt=F32), _new(T, D), _new(T, 4, dt=F32)
        self.dx, self.dy, self.dyk, self.dw, self.dl = _new(T, D, dt=F32), _new(T, D), _new(T * k, D), _new(T, k, dt=F32), _new(T, E, dt=F32)

    def run(self):
        self.router.forward(self.logits, self.ids, self.w)
        self.combine.forward(self.yk, self.w, self.yc)
        self.norm.forward(self.x, self.yc, self.r, self.h, self.stats)
        self.norm.backward(self.r, self.yc, self.dr, self.dh, self.dx, self.dy, self.stats, accumulate=False)
        self.combine.backward(self.dy, self.yk, self.w, self.dyk, self.dw)
        self.router.backward(self.logits, self.ids, self.dw, self.dl)
        self.opt.step(None, None, scalars=self.scalars)

    def results(self):
        return [t.clone() for t in (self.ids, self.w, self.yc, self.r, self.h, self.dx, self.dy, self.dyk, self.dw, self.dl, *self.norm.params.values(), self.opt.m, self.opt.v)]

    def wipe(self):
        for t in (self.w, self.yc, self.r, self.h, self.stats, self.dx, self.dy, self.dyk, self.dw, self.dl):
            t.fill_(math.nan)


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_on_another_stream():
    a, b = Chain(), Chain()
    a.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b.run()
    torch.cuda.current_stream().wait_stream(s)
    assert _same(a.results(), b.results())


def test_captured_and_replayed():
    """every replay against the eager result, with new inputs and new scalars put in place between them"""
    a, b = Chain(), Chain()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        b.run()
    for t in range(1, 5):
        g = torch.Generator(device=DEV).manual_seed(100 + t)
        for name in ("x", "logits", "dr"):
            v = torch.randn(getattr(a, name).shape, generator=g, device=DEV)
            getattr(a, name).copy_(v)
            getattr(b, name).copy_(v)
        sc = RtpAdamW.scalars_of(1e-2, t)
        a.scalars.copy_(sc)
        b.scalars.copy_(sc)
        a.wipe()
        b.wipe()
        a.run()
        graph.replay()
        torch.cuda.synchronize()
        assert _same(a.results(), b.results()), t


def test_two_graphs_at_once_share_nothing():
    a, b, c, d = Chain(seed=1), Chain(seed=2), Chain(seed=1), Chain(seed=2)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    graphs = []
    for s, q in ((s1, a), (s2, b)):
        s.wait_stream(torch.cuda.current_stream())
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=s):
            q.run()
        graphs.append(gr)
    for t in range(3):
        for s, gr in zip((s1, s2), graphs):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                gr.replay()
        for s in (s1, s2):
            torch.cuda.current_stream().wait_stream(s)
        c.run()
        d.run()
        torch.cuda.synchronize()
        assert _same(a.results(), c.results()) and _same(b.results(), d.results()), t


def test_creating_an_optimizer_while_capturing_is_refused():
    p, g = torch.zeros(10, device=DEV), torch.zeros(10, device=DEV)
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        p.add_(1.0)
        with pytest.raises(B.RtpError):
            RtpAdamW([dict(param=p, grad=g)], moments=None)
    graph.replay()
    torch.cuda.synchronize()
    assert (p == 1).all()
