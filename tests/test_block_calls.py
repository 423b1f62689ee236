"""What the calls around a unit refuse, on the host: nothing reaches the device, so these run without one (the addresses are never
looked at).  And the pure host functions of the optimizer."""
import ctypes as C
import math

import pytest
import torch

from paper_2311_01635_amd import RtpAdamW, RtpCombine, RtpNorm, RtpRouter
from paper_2311_01635_amd import binding as B

P = 0x10000          # an address that is a multiple of anything


def _route(**kw):
    d = B.rtp_route_desc()
    v = dict(T=4, E=16, k=2, score=0, renormalise=1, scale=1.0, groups=1, kept_groups=1, group_top=1, dtype=B.RTP_F32, grad_dtype=B.RTP_F32, ld=0, ld_grad=0)
    v.update(kw)
    for k, x in v.items():
        setattr(d, k, x)
    return d


ROUTE_BAD = [(dict(score=2), B.RTP_ERR_INVALID), (dict(dtype=3), B.RTP_ERR_INVALID), (dict(scale=math.nan), B.RTP_ERR_INVALID),
             (dict(T=-1), B.RTP_ERR_SHAPE), (dict(T=1 << 32), B.RTP_ERR_SHAPE), (dict(E=0), B.RTP_ERR_SHAPE), (dict(k=0), B.RTP_ERR_SHAPE), (dict(k=17), B.RTP_ERR_SHAPE),
             (dict(E=1025), B.RTP_ERR_UNSUPPORTED), (dict(E=64, k=33), B.RTP_ERR_UNSUPPORTED), (dict(E=130, groups=65, kept_groups=65), B.RTP_ERR_UNSUPPORTED),
             (dict(groups=3), B.RTP_ERR_SHAPE), (dict(groups=4, kept_groups=5), B.RTP_ERR_SHAPE), (dict(groups=8, kept_groups=1, k=3), B.RTP_ERR_SHAPE),
             (dict(group_top=3), B.RTP_ERR_INVALID), (dict(ld=15), B.RTP_ERR_SHAPE), (dict(ld=-16), B.RTP_ERR_SHAPE)]


@pytest.mark.parametrize("bad,status", ROUTE_BAD)
def test_route_refuses(bad, status):
    assert B.lib.rtp_route_fwd(C.byref(_route(**bad)), P, None, P + 64, P + 128, None) == status
    assert B.lib.rtp_route_bwd(C.byref(_route(**bad)), P, P + 64, P + 128, P + 256, None) == status
    assert b"rtp_route_bwd" in B.lib.rtp_last_error()


def test_route_refuses_pointers():
    f, b, d = B.lib.rtp_route_fwd, B.lib.rtp_route_bwd, _route()
    assert f(None, P, None, P, P, None) == B.RTP_ERR_INVALID
    for args in ((None, None, P, P), (P, None, None, P), (P, None, P, None)):
        assert f(C.byref(d), *args, None) == B.RTP_ERR_INVALID
    for args in ((P + 2, None, P, P), (P, P + 1, P, P), (P, None, P + 2, P), (P, None, P, P + 2)):
        assert f(C.byref(d), *args, None) == B.RTP_ERR_SHAPE
    assert b(C.byref(d), P, P, P, None, None) == B.RTP_ERR_INVALID
    assert b(C.byref(d), P, P + 64, P + 128, P, None) == B.RTP_ERR_INVALID            # the gradient over the logits
    assert b(C.byref(_route(grad_dtype=7)), P, P + 64, P + 128, P + 256, None) == B.RTP_ERR_INVALID
    assert b(C.byref(_route(ld_grad=3)), P, P + 64, P + 128, P + 256, None) == B.RTP_ERR_SHAPE
    assert f(C.byref(_route(T=0)), None, None, None, None, None) == B.RTP_OK          # no tokens: nothing to do


def test_combine_refuses():
    f, b = B.lib.rtp_combine_fwd, B.lib.rtp_combine_bwd
    ok = dict(T=4, k=2, D=8, dtype=B.RTP_BF16)
    for bad, st in ((dict(dtype=5), B.RTP_ERR_INVALID), (dict(T=-1), B.RTP_ERR_SHAPE), (dict(T=1 << 31), B.RTP_ERR_SHAPE), (dict(k=0), B.RTP_ERR_SHAPE),
                    (dict(k=33), B.RTP_ERR_UNSUPPORTED), (dict(D=0), B.RTP_ERR_SHAPE), (dict(D=(1 << 20) + 1), B.RTP_ERR_SHAPE)):
        v = {**ok, **bad}
        assert f(v["T"], v["k"], v["D"], v["dtype"], P, 0, P + 4096, P + 8192, 0, None) == st
        assert b(v["T"], v["k"], v["D"], v["dtype"], P, 0, P + 1024, 0, P + 4096, P + 8192, 0, P + 9000, None) == st
    v = tuple(ok.values())
    assert f(*v, P, 7, P + 4096, P + 8192, 0, None) == B.RTP_ERR_SHAPE
    assert f(*v, P + 1, 0, P + 4096, P + 8192, 0, None) == B.RTP_ERR_SHAPE
    assert f(*v, P, 0, P + 4098, P + 8192, 0, None) == B.RTP_ERR_SHAPE
    assert f(*v, None, 0, P, P, 0, None) == B.RTP_ERR_INVALID
    assert f(*v, P, 0, None, P, 0, None) == B.RTP_ERR_INVALID                         # in place
    assert b(*v, P, 0, None, 0, P, P + 8192, 0, P + 9000, None) == B.RTP_ERR_INVALID   # dweights needs Yk
    assert b(*v, P, 0, P + 512, 0, P, P + 512, 0, None, None) == B.RTP_ERR_INVALID
    assert b(*v, None, 0, None, 0, None, None, 0, None, None) == B.RTP_OK             # nothing asked for
    assert f(0, 2, 8, B.RTP_BF16, None, 0, None, None, 0, None) == B.RTP_OK


def _norm(**kw):
    d = B.rtp_norm_desc()
    v = dict(T=4, D=8, kind=0, parts=B.RTP_NORM_JOIN | B.RTP_NORM_POST | B.RTP_NORM_PRE, gate=0, stream_dtype=B.RTP_BF16, dtype=B.RTP_BF16, eps=1e-5,
             res_scale=1.0, out_scale=1.0)
    v.update(kw)
    for k, x in v.items():
        setattr(d, k, x)
    return d


def _io(**kw):
    io = B.rtp_norm_io()
    for i, n in enumerate(("x_dev", "y_dev", "r_dev", "h_dev", "stats_dev")):
        setattr(io, n, P * (i + 1))
    for k, x in kw.items():
        setattr(io, k, x)
    return io


def _grads(**kw):
    g = B.rtp_norm_grads()
    for i, n in enumerate(("r_dev", "y_dev", "dr_dev", "dh_dev", "stats_dev", "dx_dev", "dy_dev")):
        setattr(g, n, P * (i + 1))
    for k, x in kw.items():
        setattr(g, k, x)
    return g


NORM_BAD = [(dict(kind=2), B.RTP_ERR_INVALID), (dict(dtype=9), B.RTP_ERR_INVALID), (dict(stream_dtype=B.RTP_F16), B.RTP_ERR_UNSUPPORTED),
            (dict(parts=0), B.RTP_ERR_INVALID), (dict(parts=8 | 1), B.RTP_ERR_INVALID), (dict(parts=B.RTP_NORM_POST | B.RTP_NORM_PRE), B.RTP_ERR_INVALID),
            (dict(gate=3), B.RTP_ERR_INVALID), (dict(gate=1, gate_dev=P, parts=B.RTP_NORM_PRE), B.RTP_ERR_INVALID), (dict(gate=1), B.RTP_ERR_INVALID),
            (dict(T=-1), B.RTP_ERR_SHAPE), (dict(D=0), B.RTP_ERR_SHAPE), (dict(D=(1 << 20) + 1), B.RTP_ERR_SHAPE), (dict(eps=0.0), B.RTP_ERR_INVALID),
            (dict(eps=math.nan), B.RTP_ERR_INVALID), (dict(res_scale=math.inf), B.RTP_ERR_INVALID), (dict(out_scale=math.nan), B.RTP_ERR_INVALID),
            (dict(gate=2, gate_dev=P * 20, ld_gate=7), B.RTP_ERR_SHAPE), (dict(w_post_dev=P + 2), B.RTP_ERR_SHAPE), (dict(gate=2, gate_dev=P + 1), B.RTP_ERR_SHAPE)]


@pytest.mark.parametrize("bad,status", NORM_BAD)
def test_norm_refuses(bad, status):
    assert B.lib.rtp_norm_fwd(C.byref(_norm(**bad)), C.byref(_io()), None) == status
    assert B.lib.rtp_norm_bwd(C.byref(_norm(**bad)), C.byref(_grads()), None) == status
    assert (B.lib.rtp_norm_ws_bytes(C.byref(_norm(**bad))) == 0) == (bad not in (dict(gate=1), dict(w_post_dev=P + 2), dict(gate=2, gate_dev=P + 1)))


def test_norm_refuses_pointers():
    f, b, d = B.lib.rtp_norm_fwd, B.lib.rtp_norm_bwd, _norm()
    for n in ("x_dev", "y_dev", "r_dev", "h_dev", "stats_dev"):
        assert f(C.byref(d), C.byref(_io(**{n: None})), None) == B.RTP_ERR_INVALID, n
        assert f(C.byref(d), C.byref(_io(**{n: P * 9 + 1})), None) == B.RTP_ERR_SHAPE, n
    for n in ("ld_x", "ld_y", "ld_r", "ld_h"):
        assert f(C.byref(d), C.byref(_io(**{n: 7})), None) == B.RTP_ERR_SHAPE, n
    for over in (dict(r_dev=P * 2), dict(h_dev=P), dict(h_dev=P * 2), dict(h_dev=P * 3), dict(r_dev=P, ld_r=16)):
        assert f(C.byref(d), C.byref(_io(**over)), None) == B.RTP_ERR_INVALID, over
    for n in ("r_dev", "y_dev", "dh_dev", "stats_dev", "dx_dev", "dy_dev"):
        assert b(C.byref(d), C.byref(_grads(**{n: None})), None) == B.RTP_ERR_INVALID, n
        assert b(C.byref(d), C.byref(_grads(**{n: P * 9 + 1})), None) == B.RTP_ERR_SHAPE, n
    for over in (dict(dx_dev=P), dict(dx_dev=P * 2), dict(dx_dev=P * 3, ld_dr=16), dict(dy_dev=P * 2), dict(dy_dev=P * 4), dict(dy_dev=P * 6)):
        assert b(C.byref(d), C.byref(_grads(**over)), None) == B.RTP_ERR_INVALID, over
    assert b(C.byref(_norm(parts=B.RTP_NORM_JOIN)), C.byref(_grads(dr_dev=None)), None) == B.RTP_ERR_INVALID     # no gradient at all
    # sums over rows need a workspace of their own
    need = B.lib.rtp_norm_ws_bytes(C.byref(d))
    assert need > 0
    for ws in (dict(), dict(ws_dev=P * 10 + 8, ws_bytes=1 << 30)):
        assert b(C.byref(d), C.byref(_grads(dw_pre_dev=P * 9, **ws)), None) == B.RTP_ERR_INVALID
    assert b(C.byref(d), C.byref(_grads(dw_pre_dev=P * 9, dw_post_dev=P * 8, ws_dev=P * 10, ws_bytes=15)), None) == B.RTP_ERR_SHAPE
    assert f(C.byref(_norm(T=0)), C.byref(B.rtp_norm_io()), None) == B.RTP_OK
    assert b(C.byref(_norm(T=0)), C.byref(B.rtp_norm_grads()), None) == B.RTP_OK


def _tensors(*spans, dtype=B.RTP_BF16, master=0, **kw):
    arr = (B.rtp_adamw_tensor * max(len(spans), 1))()
    for i, (e, n) in enumerate(zip(arr, spans)):
        e.param_dev, e.grad_dev, e.numel, e.dtype = P * (1000 + 300 * i), P * (5000 + 300 * i), n, dtype
        e.master_dev = P * (9000 + 300 * i) if master else None
        for k, x in kw.items():
            setattr(e, k, x)
    return arr


def _adamw(arr, n, **kw):
    d = B.rtp_adamw_desc()
    d.tensors, d.count, d.moments, d.m_dev, d.v_dev, d.exps_dev, d.table_dev = arr, n, B.RTP_MOMENTS_8BIT, P * 20000, P * 30000, P * 40000, P * 50000
    for k, x in kw.items():
        setattr(d, k, x)
    h = C.c_void_p()
    st = B.lib.rtp_adamw_create(C.byref(h), C.byref(d))
    assert not h
    return st


def test_adamw_refuses():
    t = _tensors(1000, 7)
    assert B.lib.rtp_adamw_blocks(t, 2) == 5 and B.lib.rtp_adamw_table_bytes(t, 2) > 0
    assert B.lib.rtp_adamw_blocks(None, 2) == -1 and B.lib.rtp_adamw_blocks(t, 0) == -1 and B.lib.rtp_adamw_table_bytes(_tensors(0), 1) == 0
    for bad in (dict(m_dev=None), dict(v_dev=None), dict(exps_dev=None), dict(table_dev=None), dict(moments=2)):
        assert _adamw(t, 2, **bad) == B.RTP_ERR_INVALID, bad
    for bad in (dict(m_dev=P + 8), dict(table_dev=P + 4), dict(exps_dev=P + 1), dict(tensors=None), dict(count=0)):
        assert _adamw(t, 2, **bad) == B.RTP_ERR_SHAPE, bad
    for bad, st in ((dict(param_dev=None), B.RTP_ERR_INVALID), (dict(grad_dev=None), B.RTP_ERR_INVALID), (dict(dtype=4), B.RTP_ERR_INVALID),
                    (dict(weight_decay=math.nan), B.RTP_ERR_INVALID), (dict(param_dev=P + 1), B.RTP_ERR_SHAPE), (dict(grad_dev=P + 2), B.RTP_ERR_SHAPE),
                    (dict(numel=0), B.RTP_ERR_SHAPE), (dict(numel=-5), B.RTP_ERR_SHAPE)):
        assert _adamw(_tensors(1000, **bad), 1) == st, bad
    assert _adamw(_tensors(1000, dtype=B.RTP_F32, master=1), 1) == B.RTP_ERR_INVALID


def test_adamw_refuses_memory_that_overlaps():
    def two_at(**kw):
        t = _tensors(1000, 1000, master=1)
        for k, x in kw.items():
            setattr(t[1], k, x)
        return t
    first = _tensors(1000, 1000, master=1)[0]
    for kw in (dict(param_dev=first.param_dev), dict(param_dev=first.param_dev + 1998), dict(param_dev=first.grad_dev + 64), dict(master_dev=first.master_dev),
               dict(grad_dev=first.param_dev), dict(master_dev=P * 20000), dict(param_dev=P * 30000 + 254), dict(grad_dev=P * 50000)):
        assert _adamw(two_at(**kw), 2) == B.RTP_ERR_INVALID, kw
        assert b"overlaps" in B.lib.rtp_last_error()
    assert _adamw(_tensors(1000), 1, v_dev=P * 20000) == B.RTP_ERR_INVALID


def test_adamw_step_refuses():
    h, sc = B.rtp_adamw_hyper(1e-3, 0.9, 0.999, 1e-8, 1, 0), B.rtp_adamw_scalars()
    assert B.lib.rtp_adamw_step(None, C.byref(h), None, None, None) == B.RTP_ERR_INVALID
    assert B.lib.rtp_adamw_moments(None, B.RTP_F32, P, P, None) == B.RTP_ERR_INVALID
    for bad in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=1e-60), dict(lr=math.inf), dict(step=0)):
        g = B.rtp_adamw_hyper(1e-3, 0.9, 0.999, 1e-8, 1, 0)
        for k, x in bad.items():
            setattr(g, k, x)
        assert B.lib.rtp_adamw_scalars_of(C.byref(g), C.byref(sc)) == B.RTP_ERR_INVALID, bad
    assert B.lib.rtp_adamw_destroy(None) == B.RTP_OK


@pytest.mark.parametrize("step", [1, 2, 1000, 10 ** 7])
def test_adamw_scalars(step):
    h, sc = B.rtp_adamw_hyper(1e-3, 0.9, 0.999, 1e-8, step, 0xDEADBEEF), B.rtp_adamw_scalars()
    assert B.lib.rtp_adamw_scalars_of(C.byref(h), C.byref(sc)) == B.RTP_OK
    # each is one rounding to fp32 (2^-24) of what 64 bits give
    for got, want in ((sc.beta1, 0.9), (sc.one_minus_beta1, 0.1), (sc.beta2, 0.999), (sc.one_minus_beta2, 0.001), (sc.lr, 1e-3), (sc.eps, 1e-8),
                      (sc.step_size, 1e-3 / (1 - 0.9 ** step)), (sc.root_scale, 1 / math.sqrt(1 - 0.999 ** step))):
        assert abs(got - want) <= 2.0 ** -24 * want * 1.001
    assert sc.seed == 0xDEADBEEF


def test_python_checks():
    t = torch.zeros
    with pytest.raises(ValueError):
        RtpRouter(8, 2, score="tanh")
    with pytest.raises(B.RtpError):
        RtpRouter(8, 9)
    with pytest.raises(B.RtpError):
        RtpRouter(8, 2, groups=3)
    with pytest.raises(ValueError):
        RtpRouter(8, 2).forward(t(4, 8), t(4, 2, dtype=torch.int32), t(4, 2))         # not on the GPU
    with pytest.raises(ValueError):
        RtpCombine(33)
    with pytest.raises(ValueError):
        RtpCombine(2).forward(t(8, 8), None, t(4, 8))
    with pytest.raises(ValueError):
        RtpNorm(8, kind="batch")
    with pytest.raises(ValueError):
        RtpNorm(8, post=False, w_post=t(8))
    with pytest.raises(ValueError):
        RtpNorm(8, w_pre=t(8))                                                        # a parameter that is not on the GPU
    with pytest.raises(B.RtpError):
        RtpNorm(8, join=False, pre=False)
    with pytest.raises(B.RtpError):
        RtpNorm(8, eps=-1.0)
    with pytest.raises(B.RtpError):
        RtpNorm(8, stream_dtype=torch.float16, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        RtpAdamW([], "f32")
    with pytest.raises(ValueError):
        RtpAdamW([dict(param=t(8), grad=t(8))])
    with pytest.raises(ValueError):
        RtpAdamW([dict(param=t(8), grad=t(8))], state="4bit")
