"""Several AdamW steps with the moments of the plain form bit for bit: m = beta1 m + (1 - beta1) g and v = beta2 v + (1 - beta2) g^2 with
every product and sum rounded to fp32 by itself.  Half a unit of fp32 is no error of one step, but with 8-bit moments it decides a
random rounding whose result the next steps go on from."""
import pytest
import torch

import block_reference as ref
from paper_2311_01635_amd import RtpAdamW

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
B1, B2, LR, EPS = 0.9, 0.999, 1e-3, 1e-8
LARGE, SMALL = [1, 255, 257, 4097, 4_000_003], [1, 300, 5000]


def encode(x, top, bits):
    """(codes, exponents, the numbers they stand for) of whole blocks, from the format's definition in 64 bits"""
    a = x.abs().double()
    E = (ref.binade(x.abs().view(-1, ref.BLOCK).amax(1)) + 127).clamp(min=1)
    base = (E - 127).repeat_interleave(ref.BLOCK)
    # the binade whose eighths it is rounded to (zero has none of its own)
    e = torch.maximum(torch.where(a > 0, torch.frexp(a).exponent - 1, -1000).to(torch.int64), base - (top - 1))
    n = torch.floor(a * ref.two(3 - e) + bits.double() / 65536.0)
    if top == ref.TOP_V:
        n = torch.where(a > 0, n.clamp_min(1), n)
    # eighths count on through the binades: 8 to 15 are a binade's own, below 8 is the last one's denormal part
    code = (8 * (e - base + top - 1) + n).to(torch.int64)
    value = n * ref.two(e - 3)
    if top == ref.TOP_M:
        code = torch.where(x < 0, code + 128, code)
        value = torch.where(x < 0, -value, value)
    return code.to(torch.uint8), E.to(torch.uint8), value.float()


@pytest.mark.parametrize("state,dtype,master,sizes,steps", [("8bit", F32, False, LARGE, 8), ("f32", F32, False, LARGE, 3), ("8bit", BF16, False, SMALL, 5), ("8bit", BF16, True, SMALL, 5),
                                                            ("8bit", F16, False, SMALL, 5), ("f32", F16, True, SMALL, 3)])
def test_moments_of_several_steps(state, dtype, master, sizes, steps):
    byte = state == "8bit"
    gen = torch.Generator(device=DEV).manual_seed(11)
    blocks = [-(-n // ref.BLOCK) for n in sizes]
    N = sum(blocks) * ref.BLOCK
    live, spans, at = torch.zeros(N, dtype=torch.bool, device=DEV), [], 0
    for n, b in zip(sizes, blocks):
        live[at:at + n] = True
        spans.append((at, n))
        at += b * ref.BLOCK
    params = [(0.02 * torch.randn(n, generator=gen, device=DEV)).to(dtype) for n in sizes]
    copies = [p.float() for p in params]
    grads = [torch.empty(n, device=DEV) for n in sizes]
    # gradients of blocks differ in size; some elements never have one, in blocks where others do: their moments stay exact zeros
    size = (1e-3 * torch.exp(torch.randn(N // ref.BLOCK, generator=gen, device=DEV))).repeat_interleave(ref.BLOCK)
    size = size * live * (torch.rand(N, generator=gen, device=DEV) >= 0.1)
    opt = RtpAdamW([dict(param=p, grad=g, weight_decay=0.1, **(dict(master=c) if master else {})) for p, g, c in zip(params, grads, copies)], state)
    clip = torch.full((1,), 0.7, device=DEV)
    b1, c1, b2, c2 = (torch.tensor(x, dtype=F32, device=DEV) for x in (B1, 1 - B1, B2, 1 - B2))
    m = v = torch.zeros(N, device=DEV)
    place = torch.arange(N, device=DEV)
    for t in range(1, steps + 1):
        g = torch.randn(N, generator=gen, device=DEV) * size
        for (a, n), to in zip(spans, grads):
            to.copy_(g[a:a + n])
        before = [(c if master else p).double() for p, c in zip(params, copies)]
        seed = 0x51ED270B * t & ref.MASK
        opt.step(LR, t, betas=(B1, B2), eps=EPS, seed=seed, grad_scale=clip)
        g = g * clip
        m, v = b1 * m + c1 * g, b2 * v + c2 * (g * g)
        d = LR / (1 - B1 ** t) * m.double() / (torch.sqrt(v.double() / (1 - B2 ** t)) + EPS)
        if byte:
            rm, rv, _ = ref.random_bits(place, seed)
            (mc, em, m), (vc, ev, v) = encode(m, ref.TOP_M, rm), encode(v, ref.TOP_V, rv)
            assert torch.equal(opt.exps[:, 0], em) and torch.equal(opt.exps[:, 1], ev), t
            assert int((opt.m != mc)[live].sum()) == 0 and int((opt.v != vc)[live].sum()) == 0, t
            assert torch.equal(opt.moments(F32)[0][live], m[live]) and torch.equal(opt.moments(F32)[1][live], v[live])
        else:
            assert torch.equal(opt.m[live], m[live]) and torch.equal(opt.v[live], v[live]), t
        # the parameter: 3 u of itself, and 24 u of its update (a root, a quotient, the host's rounded factors).  Rounded at random it is a
        # neighbour, one spacing away at most: 2^-7 (bf16) or 2^-10 (fp16, and its smallest spacing)
        step = 0.0 if dtype == F32 or master else torch.finfo(dtype).eps
        for (a, n), p, c, p0 in zip(spans, params, copies, before):
            got, want = (c if master else p).double(), p0 * (1 - LR * 0.1) - d[a:a + n]
            tol = (3 * U + step) * (want.abs() + p0.abs()) + 24 * U * d[a:a + n].abs() + (2.0 ** -24 if step and dtype == F16 else 0)
            assert ((got - want).abs() <= tol).all(), t
            if master:
                assert torch.equal(p, c.to(dtype))
    opt.close()
