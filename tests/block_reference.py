"""The operators around a unit, from their definitions in 64 bits (torch, CPU or GPU).  Written for the tests alone; shares nothing
with the kernels."""
import math

import torch


# ---- router -----------------------------------------------------------------------------------------------------------

def scores(logits, score):
    """softmax or sigmoid of [T, E] logits; an expert whose logit is -infinity has 0."""
    l = logits.double()
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-l))
    shut = l == -math.inf
    return torch.softmax(torch.where(shut.all(1, keepdim=True), 0.0, l), 1) * ~shut


def route(logits, k, score="softmax", renorm=True, scale=1.0, groups=1, kept=1, group_top=1, bias=None):
    """(ids, weights) row by row, with sorts of Python's (stable: equal ones stay in the order of their index)."""
    p = scores(logits, score)
    ids, weights = [], []
    for l, s in zip(logits.double().tolist(), p.tolist()):
        E = len(l)
        if bias is None and groups == 1:
            choice = list(l)
        else:
            choice = [-math.inf if x == -math.inf else v + (0.0 if bias is None else b) for x, v, b in zip(l, s, [0.0] * E if bias is None else bias.double().tolist())]
        eligible = list(range(E))
        if groups > 1:
            n = E // groups
            def of(g):
                best = sorted(choice[g * n:(g + 1) * n], reverse=True)
                return best[0] + (best[1] if group_top == 2 and n > 1 and best[1] > -math.inf else 0.0)
            best = sorted(range(groups), key=lambda g: -of(g))[:kept]
            eligible = [e for e in range(E) if e // n in best]
        top = sorted(eligible, key=lambda e: -choice[e])[:k]
        w = weights_of([l[e] for e in top], [s[e] for e in top], score, renorm)
        ids.append(top)
        weights.append([scale * x for x in w])
    return torch.tensor(ids, dtype=torch.int32), torch.tensor(weights, dtype=torch.float64)


def weights_of(l, s, score, renorm):
    if not renorm:
        return [0.0 if x == -math.inf else v for x, v in zip(l, s)]
    # a sum of scores that underflows cancels: in logarithms
    lg = [x if score == "softmax" or x == -math.inf else -math.log1p(math.exp(-x)) if x > -500 else x for x in l]
    m = max(lg)
    if m == -math.inf:
        return [0.0] * len(l)
    e = [math.exp(x - m) for x in lg]
    return [x / sum(e) for x in e]


def route_weights(logits, ids, score, renorm, scale):
    """Differentiable: the weights of given ids (distinct, all open), for gradients by autograd."""
    l = logits
    p = torch.softmax(l, 1) if score == "softmax" else torch.sigmoid(l)
    w = p.gather(1, ids.long())
    return scale * (w / w.sum(1, keepdim=True) if renorm else w)


# ---- norms ------------------------------------------------------------------------------------------------------------

def norm(v, kind, eps, w=None, b=None):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    n = v / torch.sqrt(v.square().mean(1, keepdim=True) + eps)
    n = n if w is None else n * w
    return n if b is None else n + b


def stats(v, kind, eps):
    mu = v.mean(1) if kind == "layer" else torch.zeros_like(v[:, 0])
    return mu, 1 / torch.sqrt((v - mu[:, None]).square().mean(1) + eps)


def join(x, y, kind, eps, post, res_scale, out_scale, w=None, b=None, gate=None):
    if post:
        y = norm(y, kind, eps, w, b)
    return res_scale * x + out_scale * (y if gate is None else gate * y)


# ---- AdamW ------------------------------------------------------------------------------------------------------------

BLOCK, TOP_M, TOP_V = 256, 14, 30
MASK = 0xFFFFFFFF


def random_bits(place, seed):
    """(16 bits for m, 16 for v, 16 for the parameter) of elements at `place` (int64 tensor)."""
    x = (place * 0x9E3779B1 + seed) & MASK
    x = ((x ^ (x >> 15)) * 0xB504F333) & MASK
    x = ((x ^ (x >> 16)) * 0x243F6A89) & MASK
    x = x ^ (x >> 15)
    return x & 0xFFFF, x >> 16, ((x * 0x9E3779B1) & MASK) >> 16


def binade(x):
    """floor(log2 |x|), of at least 2^-126"""
    return torch.frexp(x.abs().clamp_min(2.0 ** -126)).exponent.to(torch.int64) - 1


def two(e):
    return torch.ldexp(torch.ones((), dtype=torch.float64), torch.as_tensor(e).double()) if not torch.is_tensor(e) else ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def spacing(x, top, mantissa=3):
    """distance between the codes around each element of x (whole blocks, flat)"""
    last = binade(x.abs().view(-1, BLOCK).amax(1)) - (top - 1)
    return two(torch.maximum(binade(x).view(-1, BLOCK), last[:, None]) - mantissa).view(-1)


def decode(codes, exps, top):
    """numbers that codes stand for, by the format's definition, code by code"""
    out = []
    for c, E in zip(codes.view(-1, BLOCK).tolist(), exps.tolist()):
        for x in c:
            sign = -1.0 if top == TOP_M and x & 128 else 1.0
            mag = x & 127 if top == TOP_M else x
            e, f = mag >> 3, mag & 7
            out.append(sign * (math.ldexp(1 + f / 8, e - top + max(E, 1) - 127) if e else math.ldexp(f / 8, 1 - top + max(E, 1) - 127)) if E < 255 else math.nan)
    return torch.tensor(out, dtype=torch.float64)


def adamw(p, g, m, v, lr, wd, step, betas=(0.9, 0.999), eps=1e-8):
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    p = p * (1 - lr * wd) - lr / (1 - betas[0] ** step) * m / (torch.sqrt(v / (1 - betas[1] ** step)) + eps)
    return p, m, v
