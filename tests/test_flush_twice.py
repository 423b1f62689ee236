"""rtp_ring_flush twice without a pass in between: the caller may have written the weight store after the first (an optimizer step), and
the second (reading the weights back, a checkpoint) leaves it as it is."""
import pytest
import torch

from paper_2311_01635_amd import binding as B

MODES = [B.RTP_DOUBLE_BUFFER, B.RTP_INPLACE_STAGED, B.RTP_INPLACE_BLOCKING]


def _pass(ring, lin, pass_, n, call):
    ring.begin(pass_)
    for t in range(n):
        if t < n - 1:
            ring.rotate_step(B.RTP_CW if pass_ == B.RTP_PASS_FWD else B.RTP_CCW, t)
        call(t)
    ring.end()


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("n", [1, 4])
def test_only_the_first_flush_copies_weights(n, mode):
    w = 16 * 8 * n * 4
    ring = B.Ring(n, n // 2, mode, w, w, flags=B.RTP_FLAG_DRY_RUN)
    lin = B.Linear(ring, 4, 8, 8 * n, B.RTP_SPLIT_OUT, B.RTP_F32)
    outs = lambda: [r for r in ring.trace(clear=True) if r[0] == "w_out" and r[2] < 0]   # noqa: E731
    for _ in range(2):
        _pass(ring, lin, B.RTP_PASS_FWD, n, lambda t: lin.fwd(t, None, None))
        ring.trace(clear=True)
        ring.flush()
        assert len(outs()) == 1
        ring.flush()
        assert not outs()
        _pass(ring, lin, B.RTP_PASS_FWD, n, lambda t: lin.fwd(t, None, None))
        _pass(ring, lin, B.RTP_PASS_BWD, n, lambda t: lin.bwd(t, None, None, None))
        ring.trace(clear=True)
        ring.flush()
        ring.zero_grads()
        ring.flush()
        assert len(outs()) == 1
    lin.close()
    ring.close()


@pytest.mark.gpu
@pytest.mark.parametrize("mode", MODES)
def test_weights_written_between_two_flushes_stay(mode):
    from paper_2311_01635_amd.layers import RtpLinear
    n, T, I, O = 4, 32, 64, 128
    layer = RtpLinear(torch.zeros(O, I), T, n, 1, mode=mode)
    X, Y = torch.ones(T, I, device="cuda:0", dtype=torch.bfloat16), torch.empty(T, O, device="cuda:0", dtype=torch.bfloat16)
    dX = torch.empty_like(X)
    layer.forward(X, Y)
    layer.backward(X, torch.ones_like(Y), dX)
    layer.ring.flush()
    layer.sync()
    layer.home_w.view(torch.bfloat16).fill_(1.0)
    torch.cuda.synchronize()
    W, _ = layer.gathered()                                  # flushes again
    assert (W == 1.0).all()
    layer.forward(X, Y)
    layer.sync()
    assert (Y == I).all()
    layer.close()
