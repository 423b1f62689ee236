"""The operators around a rotated unit in a training step, as cases that can be timed: the router that says which experts
a token goes to, the weighted combination of what they give, the norms, gate and residual around a unit, and the AdamW
step over the ring stores.

A case is a dict of plain values; `prepare` makes what a program has in hand before the call, `run` makes one call:
the framework's kernels where `own` is true, else the same in elementary torch operations.  `exact` is the
operator's definition in 64 bits.

Random rounding (AdamW with 8-bit states, 16-bit weights without a master copy) draws its bits from a seed and the element's
place, so that both forms round alike.
"""
import math

import torch

own = False

DEV = "cuda:0"
_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_ES = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 256                    # elements of an 8-bit state that share an exponent
TOP_M, TOP_V = 14, 30          # exponent code of the binade that a block's largest element is in
BETA1, BETA2, EPS = 0.9, 0.999, 1e-8


def listed():
    return [
        # the block around a prompt's last token or two: latency alone
        dict(name="norm_decode", op="norm", dir="fwd", T=2, D=4096, kind="rms", post=True, pre=True, gate="none", bias=False, stream="bf16", block="bf16"),
        # between two Llama-7B-shaped blocks: residual stream in fp32, norm on both sides, a scale per channel
        dict(name="norm_7b_fwd", op="norm", dir="fwd", T=4096, D=4096, kind="rms", post=True, pre=True, gate="channel", bias=False, stream="f32", block="bf16"),
        # the GPT-2-small-shaped block with a batch whose sequences end where they end, gated per element
        dict(name="norm_gpt2s_ragged_bwd", op="norm", dir="bwd", T=1990, D=768, kind="layer", post=True, pre=True, gate="element", bias=True, stream="bf16", block="bf16"),
        # backward of the widest unit's surroundings
        dict(name="norm_8192_bwd", op="norm", dir="bwd", T=8192, D=8192, kind="rms", post=True, pre=True, gate="channel", bias=False, stream="bf16", block="bf16"),
        # eight experts, two a token: the expert benchmark's batch
        dict(name="route_8_fwd", op="route", dir="fwd", T=8192, E=8, k=2, score="softmax", renorm=True, groups=1, kept=1, group_top=1, bias=False, logits="f32", scale=1.0),
        # many small experts behind a balanced, grouped choice
        dict(name="route_256_grouped_fwd", op="route", dir="fwd", T=16384, E=256, k=8, score="sigmoid", renorm=True, groups=8, kept=4, group_top=2, bias=True, logits="f32", scale=2.5),
        # gradient of the scores, an odd number of experts and of tokens
        dict(name="route_150_bwd", op="route", dir="bwd", T=5003, E=150, k=6, score="softmax", renorm=False, groups=1, kept=1, group_top=1, bias=False, logits="bf16", scale=1.0),
        # outputs of two experts a token
        dict(name="combine_2_fwd", op="combine", dir="fwd", T=8192, k=2, D=4096, dtype="bf16"),
        # their gradients, eight experts a token, an odd batch
        dict(name="combine_8_bwd", op="combine", dir="bwd", T=4099, k=8, D=2048, dtype="bf16"),
        # the Llama-7B-shaped unit's eight slots, fp32 moments, bf16 weights with their fp32 copy
        dict(name="adamw_7b_unit_f32", op="adamw", tensors=8, size=16908288, mixed=False, dtype="bf16", master=True, state="f32"),
        # the same slots with 8-bit moments and no copy of the weights
        dict(name="adamw_7b_unit_8bit", op="adamw", tensors=8, size=16908288, mixed=False, dtype="bf16", master=False, state="8bit"),
        # a model's many small tensors, no size like another
        dict(name="adamw_many_8bit", op="adamw", tensors=150, size=589824, mixed=True, dtype="f32", master=False, state="8bit"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm", "route", "combine", "adamw"])
    if op == "norm":
        T, D = _log(rng, 1, 16384), _log(rng, 64, 8192)
        D = D if rng.random() < 0.3 else -(-D // 8) * 8
        stream, block = rng.choice([("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32"), ("f16", "f16")])
        kind = rng.choice(["rms", "layer"])
        return dict(op=op, dir=rng.choice(["fwd", "bwd"]), T=T, D=D, kind=kind, post=rng.random() < 0.7, pre=rng.random() < 0.8,
                    gate=rng.choice(["none", "channel", "element"]), bias=kind == "layer", stream=stream, block=block)
    if op == "route":
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * _log(rng, 4, 512 // groups)
        kept = 1 if groups == 1 else rng.randint(2, groups)
        k = rng.randint(1, min(12, E // groups * kept))
        score = rng.choice(["softmax", "sigmoid"])
        return dict(op=op, dir=rng.choice(["fwd", "bwd"]), T=_log(rng, 16, 32768), E=E, k=k, score=score, renorm=rng.random() < 0.6, groups=groups,
                    kept=kept, group_top=rng.choice([1, 2]), bias=rng.random() < 0.5, logits=rng.choice(["f32", "f32", "bf16", "f16"]),
                    scale=rng.choice([1.0, 2.5]))
    if op == "combine":
        T, k, D = _log(rng, 1, 16384), rng.randint(1, 8), _log(rng, 64, 8192)
        while T * k * D > 1 << 28:
            T = -(-T // 2)
        return dict(op=op, dir=rng.choice(["fwd", "bwd"]), T=T, k=k, D=D if rng.random() < 0.3 else -(-D // 8) * 8, dtype=rng.choice(["bf16", "f16", "f32"]))
    tensors = _log(rng, 1, 200)
    size = max(1, _log(rng, 10 ** 4, 10 ** 8) // tensors)
    dtype = rng.choice(["bf16", "f32"])
    return dict(op="adamw", tensors=tensors, size=size, mixed=rng.random() < 0.5, dtype=dtype, master=dtype != "f32" and rng.random() < 0.5,
                state=rng.choice(["f32", "8bit"]))


# ---- inputs --------------------------------------------------------------------------------------------------------

def _sizes(c):
    if not c["mixed"]:
        return [c["size"]] * c["tensors"]
    return [max(1, (c["size"] >> (i % 7)) - i * 37 % 101) for i in range(c["tensors"])]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    s = globals()["_prepare_" + case["op"]](case, gen)
    s["case"] = case
    if own:   # the objects that a program keeps: they hold sizes and pointers, nothing of the inputs' values
        import paper_2311_01635_amd as rtp
        globals()["_own_" + case["op"]](rtp, s)
    return s


def _randn(gen, *shape, scale=1.0, dtype=torch.float32, shift=0.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * scale + shift).to(dtype)


def _empty(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device=DEV)


def _prepare_norm(c, gen):
    T, D, S, B = c["T"], c["D"], _DT[c["stream"]], _DT[c["block"]]
    s = dict(w_post=_randn(gen, D, scale=0.1, shift=1.0), w_pre=_randn(gen, D, scale=0.1, shift=1.0),
             b_post=_randn(gen, D, scale=0.1), b_pre=_randn(gen, D, scale=0.1), y=_randn(gen, T, D, scale=0.5, dtype=B, shift=0.05))
    s["gate"] = (None if c["gate"] == "none" else _randn(gen, D, scale=0.2, shift=0.5) if c["gate"] == "channel" else
                 _randn(gen, T, D, scale=0.2, dtype=B, shift=0.5))
    # a residual stream's channels differ in size, a few of them by a lot
    width = torch.exp(0.5 * torch.randn(D, generator=gen, device=DEV))
    rows = _randn(gen, T, D) * width + 0.1
    s["r" if c["dir"] == "bwd" else "x"] = rows.to(S)
    s["rows"] = _empty(T, D, dtype=S)        # r (forward) or dx (backward)
    s["h"] = _empty(T, D, dtype=B)           # h or dy
    if c["dir"] == "bwd":
        s["dr"], s["dh"] = _randn(gen, T, D, scale=0.1, dtype=S), _randn(gen, T, D, scale=0.1, dtype=B)
        s["stats"] = torch.stack([*_moments(c, s["y"].double()), *_moments(c, s["r"].double())], 1).float()
        if c["gate"] == "element":
            s["dgate"] = _empty(T, D, dtype=B)
    else:
        s["stats"] = _empty(T, 4)
    return s


def _moments(c, v):
    """mean and 1 / deviation of each row, as the forward pass leaves them to the backward pass"""
    mu = v.mean(1) if c["kind"] == "layer" else v.new_zeros(v.shape[0])
    return mu, ((v - mu[:, None]).square().mean(1) + 1e-5).rsqrt()


def _prepare_route(c, gen):
    T, E, k = c["T"], c["E"], c["k"]
    # scores of a trained router: some experts liked by all; a few tokens are padding, where no expert is available, and a few
    # experts are closed to some tokens
    logits = _randn(gen, T, E) + 0.5 * torch.randn(E, generator=gen, device=DEV)
    closed = torch.rand(T, E, generator=gen, device=DEV) < 0.01
    closed |= torch.rand(T, 1, generator=gen, device=DEV) < 0.02
    logits = torch.where(closed, -math.inf, logits).to(_DT[c["logits"]])
    s = dict(logits=logits, bias=_randn(gen, E, scale=0.05) if c["bias"] else None,
             ids=_empty(T, k, dtype=torch.int32), weights=_empty(T, k))
    if c["dir"] == "bwd":
        s["ids"] = torch.topk(logits.float() + (0 if s["bias"] is None else s["bias"]), k, dim=1).indices.int()
        s["dweights"], s["dlogits"] = _randn(gen, T, k), torch.empty_like(logits)
    return s


def _prepare_combine(c, gen):
    T, k, D, dt = c["T"], c["k"], c["D"], _DT[c["dtype"]]
    s = dict(yk=_randn(gen, T * k, D, dtype=dt), weights=torch.softmax(_randn(gen, T, k), 1))
    s["weights"] *= (torch.rand(T, 1, generator=gen, device=DEV) >= 0.02)     # padding has no weight
    if c["dir"] == "fwd":
        s["y"] = _empty(T, D, dtype=dt)
    else:
        s["dy"], s["dyk"], s["dweights"] = _randn(gen, T, D, dtype=dt), _empty(T * k, D, dtype=dt), _empty(T, k)
    return s


def _prepare_adamw(c, gen):
    sizes = _sizes(c)
    blocks = [-(-n // BLOCK) for n in sizes]
    N = sum(blocks) * BLOCK
    live = torch.zeros(N, dtype=torch.bool, device=DEV)
    wd = torch.empty(sum(blocks), 1, device=DEV)
    s = dict(spans=[], step=1000, seed=int(torch.randint(1 << 31, (1,), generator=gen, device=DEV).item()))
    at = 0
    for i, (n, b) in enumerate(zip(sizes, blocks)):
        live[at:at + n] = True
        wd[at // BLOCK:at // BLOCK + b] = 0.0 if i % 4 == 3 else 0.1     # biases and norms do not decay
        s["spans"].append((at, n, 0.0 if i % 4 == 3 else 0.1))
        at += b * BLOCK
    # gradients of different tensors differ in size, and rows of an embedding that no token used have none
    size = torch.exp(_randn(gen, N // BLOCK, 1)) * 1e-3 * (torch.rand(N // BLOCK, 1, generator=gen, device=DEV) >= 0.03)
    flat = lambda t: (t.view(-1, BLOCK) * size).view(-1) * live   # noqa: E731
    w = _randn(gen, N, scale=0.02) * live
    s["wd"], s["w"], s["g"] = wd, w.to(_DT[c["dtype"]]), flat(_randn(gen, N))
    if c["master"]:
        s["master"] = w
    m, v = flat(_randn(gen, N, scale=0.3)), flat(torch.rand(N, generator=gen, device=DEV) + 0.05).square()
    s["clip"] = torch.full((1,), 0.7, device=DEV)              # what clipping by the global norm multiplies the gradients by
    if c["state"] == "f32":
        s["m"], s["v"] = m, v
    else:
        half = torch.full((N,), 1 << 15, dtype=torch.int64, device=DEV)
        (mc, me), (vc, ve) = _encode(m, TOP_M, half), _encode(v, TOP_V, half)
        s["m"], s["v"] = mc, vc
        s["exps"] = torch.stack([me, ve], 1).contiguous()
    return s


# ---- the framework's calls -----------------------------------------------------------------------------------------

def _own_norm(rtp, s):
    c = s["case"]
    s["norm"] = rtp.RtpNorm(c["D"], kind=c["kind"], eps=1e-5, join=True, res_scale=0.9, out_scale=0.7, gate=s["gate"] if c["gate"] == "channel" else None,
                            w_post=s["w_post"] if c["post"] else None, b_post=s["b_post"] if c["post"] and c["bias"] else None, post=c["post"],
                            w_pre=s["w_pre"] if c["pre"] else None, b_pre=s["b_pre"] if c["pre"] and c["bias"] else None, pre=c["pre"],
                            stream_dtype=_DT[c["stream"]], dtype=_DT[c["block"]])


def _own_route(rtp, s):
    c = s["case"]
    s["router"] = rtp.RtpRouter(c["E"], c["k"], score=c["score"], renormalise=c["renorm"], scale=c["scale"], groups=c["groups"], kept_groups=c["kept"],
                                group_top=c["group_top"], bias=s["bias"])


def _own_combine(rtp, s):
    s["combine"] = rtp.RtpCombine(s["case"]["k"])


def _own_adamw(rtp, s):
    # a flat store of whole blocks: what fills up a tensor's last block is stepped with it, as in the plain form
    whole = [(slice(a, a - (-n // BLOCK) * BLOCK), wd) for a, n, wd in s["spans"]]
    tensors = [dict(param=s["w"][a], grad=s["g"][a], master=s["master"][a] if "master" in s else None, weight_decay=wd) for a, wd in whole]
    s["opt"] = rtp.RtpAdamW(tensors, state=s["case"]["state"], moments=(s["m"], s["v"], s.get("exps")))


def run(s):
    return globals()["_run_" + s["case"]["op"]](s["case"], s)


def _run_norm(c, s):
    e = s["gate"] if c["gate"] == "element" else None
    if own:
        if c["dir"] == "fwd":
            s["norm"].forward(s["x"], s["y"], s["rows"], s["h"] if c["pre"] else None, s["stats"], gate=e)
            return [s["rows"], s["h"]] if c["pre"] else [s["rows"]]
        g = s["norm"].backward(s["r"], s["y"], s["dr"], s["dh"] if c["pre"] else None, s["rows"], s["h"], s["stats"], gate=e,
                               dgate=s.get("dgate"), accumulate=False)
        return {"dx": s["rows"], "dy": s["h"], **g, **({"dgate": s["dgate"]} if e is not None else {})}
    return _norm_fwd(c, s) if c["dir"] == "fwd" else _norm_bwd(c, s)


def _run_route(c, s):
    if own:
        if c["dir"] == "fwd":
            s["router"].forward(s["logits"], s["ids"], s["weights"])
            return [s["ids"], s["weights"]]
        s["router"].backward(s["logits"], s["ids"], s["dweights"], s["dlogits"])
        return s["dlogits"]
    return _route_fwd(c, s) if c["dir"] == "fwd" else _route_bwd(c, s)


def _run_combine(c, s):
    if own:
        if c["dir"] == "fwd":
            s["combine"].forward(s["yk"], s["weights"], s["y"])
            return s["y"]
        s["combine"].backward(s["dy"], s["yk"], s["weights"], s["dyk"], s["dweights"])
        return [s["dyk"], s["dweights"]]
    T, k, D, w = c["T"], c["k"], c["D"], s["weights"][:, :, None]
    yk = s["yk"].view(T, k, D).float()
    if c["dir"] == "fwd":
        return (w * yk).sum(1).to(s["yk"].dtype)
    dy = s["dy"].float()[:, None, :]
    return [(w * dy).view(T * k, D).to(s["yk"].dtype), (dy * yk).sum(2)]


def _run_adamw(c, s):
    s["step"] += 1
    s["seed"] = (s["seed"] + 0x9E3779B9) & 0xFFFFFFFF           # another pattern every step
    lr = 1e-3
    if own:
        s["opt"].step(lr, s["step"], betas=(BETA1, BETA2), eps=EPS, seed=s["seed"], grad_scale=s["clip"])
        m, v = (s["m"], s["v"]) if c["state"] == "f32" else s["opt"].moments()
    else:
        m, v = _adamw(c, s, lr)
    return {"w": s["w"], "m": m, "v": v, **({"master": s["master"]} if "master" in s else {})}


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _plain_norm(c, v, mu, rstd, w, b):
    n = (v - mu) * rstd
    o = n * w
    return n, o + b if c["bias"] else o


def _norm_fwd(c, s):
    col = lambda v: [t[:, None] for t in _moments(c, v)]   # noqa: E731
    x, y = s["x"].float(), s["y"].float()
    if c["post"]:
        y = _plain_norm(c, y, *col(y), s["w_post"], s["b_post"])[1]
    r = (0.9 * x + 0.7 * (y if s["gate"] is None else s["gate"].float() * y)).to(s["x"].dtype)
    if not c["pre"]:
        return [r]
    v = r.float()                                           # the norm of the row as it is stored
    return [r, _plain_norm(c, v, *col(v), s["w_pre"], s["b_pre"])[1].to(s["y"].dtype)]


def _norm_back(c, n, rstd, dn):
    """gradient of a row from that of its normalised values"""
    d = dn - n * (dn * n).mean(1, keepdim=True)
    return rstd * (d - dn.mean(1, keepdim=True)) if c["kind"] == "layer" else rstd * d


def _norm_bwd(c, s):
    mu_y, rs_y, mu_r, rs_r = (t[:, None] for t in s["stats"].unbind(1))
    out, d = {}, s["dr"].float()
    if c["pre"]:
        dh = s["dh"].float()
        n = (s["r"].float() - mu_r) * rs_r
        out["w_pre"] = (dh * n).sum(0)
        if c["bias"]:
            out["b_pre"] = dh.sum(0)
        d = d + _norm_back(c, n, rs_r, dh * s["w_pre"])
    out["dx"] = (0.9 * d).to(s["r"].dtype)
    e = 0.7 * d                                             # gradient of gate * N(y)
    y = s["y"].float()
    n, o = _plain_norm(c, y, mu_y, rs_y, s["w_post"], s["b_post"]) if c["post"] else (None, y)
    if c["gate"] == "channel":
        out["gate"] = (e * o).sum(0)
    elif c["gate"] == "element":
        out["dgate"] = (e * o).to(s["y"].dtype)
    e = e if s["gate"] is None else e * s["gate"].float()
    if c["post"]:
        out["w_post"] = (e * n).sum(0)
        if c["bias"]:
            out["b_post"] = e.sum(0)
        e = _norm_back(c, n, rs_y, e * s["w_post"])
    out["dy"] = e.to(s["y"].dtype)
    return out


def _scores(c, logits):
    """scores in 64 bits: which of two near ones is larger decides a whole number"""
    l = logits.double()
    if c["score"] == "sigmoid":
        return torch.sigmoid(l)
    top = l.amax(1, keepdim=True)
    e = torch.exp(l - torch.where(top == -math.inf, 0.0, top))
    return e / e.sum(1, keepdim=True).clamp_min(1e-300)


def _route_fwd(c, s):
    T, E, k, l = c["T"], c["E"], c["k"], s["logits"].double()
    p = _scores(c, s["logits"])
    choice = l
    if s["bias"] is not None or c["groups"] > 1:
        choice = torch.where(l == -math.inf, -math.inf, p if s["bias"] is None else p + s["bias"].double())
    if c["groups"] > 1:
        best = choice.view(T, c["groups"], -1).sort(dim=2, descending=True).values
        group = best[:, :, 0]
        if c["group_top"] == 2 and best.shape[2] > 1:
            group = group + torch.where(best[:, :, 1] == -math.inf, 0.0, best[:, :, 1])
        order = group.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        keep = torch.zeros_like(group, dtype=torch.bool).scatter_(1, order, True)
        # an expert of another group ranks below one that is closed
        rank = torch.where(keep.repeat_interleave(E // c["groups"], 1), 1, 0)
        first = choice.sort(dim=1, descending=True, stable=True).indices
        ids = first.gather(1, rank.gather(1, first).sort(dim=1, descending=True, stable=True).indices)[:, :k]
    else:
        ids = choice.sort(dim=1, descending=True, stable=True).indices[:, :k]
    chosen = l.gather(1, ids)
    open_ = chosen > -math.inf
    if c["renorm"]:
        lg = chosen if c["score"] == "softmax" else torch.nn.functional.logsigmoid(chosen)
        top = lg.amax(1, keepdim=True)
        w = torch.where(open_, torch.exp(lg - torch.where(top == -math.inf, 0.0, top)), 0.0)
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    else:
        w = torch.where(open_, p.gather(1, ids), 0.0)
    return [ids.int(), (c["scale"] * w).float()]


def _route_bwd(c, s):
    ids = s["ids"].long()
    l, a, scale = s["logits"].float(), s["dweights"], c["scale"]
    chosen = l.gather(1, ids)
    open_ = chosen > -math.inf
    a = torch.where(open_, a, 0.0)
    out = torch.zeros_like(l)
    sig = torch.sigmoid(chosen)
    if c["renorm"]:
        lg = chosen if c["score"] == "softmax" else torch.nn.functional.logsigmoid(chosen)
        top = lg.amax(1, keepdim=True)
        q = torch.where(open_, torch.exp(lg - torch.where(top == -math.inf, 0.0, top)), 0.0)
        q = q / q.sum(1, keepdim=True).clamp_min(1e-30)
        d = scale * q * (a - (q * a).sum(1, keepdim=True))
        out.scatter_(1, ids, d if c["score"] == "softmax" else d * (1 - sig))
    elif c["score"] == "sigmoid":
        out.scatter_(1, ids, scale * sig * (1 - sig) * a)
    else:
        p = _scores(c, s["logits"]).float()
        out.scatter_(1, ids, a)
        out = scale * p * (out - (p.gather(1, ids) * a).sum(1, keepdim=True))
    return out.to(s["logits"].dtype)


def _bits(seed, n):
    """32 random bits for each element, and 16 more: of the seed and the element's place alone (32-bit arithmetic held in 64)"""
    M = 0xFFFFFFFF
    x = (torch.arange(n, device=DEV) * 0x9E3779B1 + seed) & M
    x = x ^ (x >> 15)
    x = (x * 0xB504F333) & M
    x = x ^ (x >> 16)
    x = (x * 0x243F6A89) & M
    x = x ^ (x >> 15)
    return x & 0xFFFF, x >> 16, ((x * 0x9E3779B1) & M) >> 16


def _two(e):
    """2 to the power of whole numbers, exactly"""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _encode(x, top, rnd):
    """magnitudes (and sign, where it has one: `top` of m) in 8 bits: codes, and an exponent for each block.

    The block's largest element has exponent code `top`; below it a code is a small float with 3 bits of mantissa.
    code = floor(position + rnd / 65536): a value between two codes goes up with a probability that is its place between them."""
    a = x.abs().view(-1, BLOCK)
    E = (a.amax(1).view(torch.int32) >> 23).clamp(min=1)
    q = a.double() * _two(127 - E)[:, None]
    ee = (torch.frexp(q).exponent - 1).clamp(min=1 - top)
    code = torch.floor((ee + (top - 1)) * 8 + q * _two(3 - ee) + rnd.view(-1, BLOCK) / 65536.0).to(torch.int64)
    if top == TOP_M:
        code = torch.where((x < 0).view(-1, BLOCK), code + 128, code)
    else:
        code = torch.where((a > 0) & (code == 0), 1, code)          # a second moment that is there does not vanish
    return code.to(torch.uint8).view(-1), E.to(torch.uint8)


def _decode(codes, E, top):
    c = codes.to(torch.int32).view(-1, BLOCK)
    mag = c & 127 if top == TOP_M else c
    ee = (mag >> 3).clamp(min=1)
    frac = (mag & 7) + torch.where(mag >= 8, 8, 0)
    v = frac.double() * _two(ee - 3 - top + (E.to(torch.int32) - 127)[:, None])
    return (torch.where(c >= 128, -v, v) if top == TOP_M else v).view(-1)


def _adamw(c, s, lr):
    step, byte = s["step"], c["state"] == "8bit"
    g = s["g"] * s["clip"]
    m, v = (_decode(s["m"], s["exps"][:, 0], TOP_M).float(), _decode(s["v"], s["exps"][:, 1], TOP_V).float()) if byte else (s["m"], s["v"])
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * (g * g)
    p = (s["master"] if c["master"] else s["w"].float()).view(-1, BLOCK)
    p = p * (1 - lr * s["wd"])
    d = m / (v.sqrt() * (1 / math.sqrt(1 - BETA2 ** step)) + EPS)
    p = p.view(-1) - lr / (1 - BETA1 ** step) * d
    rnd = _bits(s["seed"], p.numel()) if byte or (c["dtype"] != "f32" and not c["master"]) else None
    if c["master"]:
        s["master"].copy_(p)
    if c["dtype"] == "f32" or c["master"]:
        s["w"].copy_(p)
    else:
        s["w"].copy_((((p.view(torch.int32).long() + rnd[2]) >> 16) << 16).int().view(torch.float32))
    if not byte:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return s["m"], s["v"]
    (mc, me), (vc, ve) = _encode(m, TOP_M, rnd[0]), _encode(v, TOP_V, rnd[1])
    s["m"].copy_(mc)
    s["v"].copy_(vc)
    s["exps"].copy_(torch.stack([me, ve], 1))
    # (a code times a power of two: bfloat16 holds it whole)
    return _decode(s["m"], me, TOP_M).bfloat16(), _decode(s["v"], ve, TOP_V).bfloat16()


# ---- what an operator cannot do without ----------------------------------------------------------------------------

def work(c):
    if c["op"] == "norm":
        n, S, B = c["T"] * c["D"], _ES[c["stream"]], _ES[c["block"]]
        e = B * n if c["gate"] == "element" else 0
        if c["dir"] == "fwd":
            return {"bytes": n * (2 * S + B + (B if c["pre"] else 0)) + e + 16 * c["T"], "flops": 12 * n}
        read = n * S + (n * B if c["post"] or c["gate"] != "none" else 0) + (n * (S + B) if c["pre"] else 0)     # dr; y; r, dh
        return {"bytes": read + n * (S + B) + 2 * e + 16 * c["T"], "flops": 30 * n}
    if c["op"] == "route":
        n = c["T"] * c["E"] * _ES[c["logits"]]
        return {"bytes": n * (1 if c["dir"] == "fwd" else 2) + c["T"] * c["k"] * 8 + 4 * c["E"], "flops": c["T"] * c["E"] * 8}
    if c["op"] == "combine":
        n, es = c["T"] * c["D"], _ES[c["dtype"]]
        slots = n * c["k"] * es
        return {"bytes": (slots if c["dir"] == "fwd" else 2 * slots) + n * es + 4 * c["T"] * c["k"], "flops": 2 * n * c["k"]}
    n, es = sum(_sizes(c)), _ES[c["dtype"]]
    weights = 2 * es if not c["master"] else es + 8
    state = 16 if c["state"] == "f32" else 4 + 4                          # in 8 bits, the moments are handed out in 16 too
    return {"bytes": n * (4 + weights + state), "flops": 16 * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    return globals()["_exact_" + case["op"]](case, s)


def _exact_norm(c, s):
    f = lambda k: None if s.get(k) is None else s[k].double()   # noqa: E731

    def centred(v):
        mu, rs = (t[:, None] for t in _moments(c, v))
        return (v - mu) * rs, rs

    y, w2, b2, w1, b1, gate = (f(k) for k in ("y", "w_post", "b_post", "w_pre", "b_pre", "gate"))
    gate = 1.0 if gate is None else gate
    ny, ry = centred(y) if c["post"] else (y, None)
    oy = (ny * w2 + (b2 if c["bias"] else 0)) if c["post"] else y
    if c["dir"] == "fwd":
        r = 0.9 * f("x") + 0.7 * gate * oy
        return [r, centred(r)[0] * w1 + (b1 if c["bias"] else 0)] if c["pre"] else [r]
    out, D, layer = {}, c["D"], c["kind"] == "layer"
    d = f("dr")
    if c["pre"]:
        nr, rr = centred(f("r"))
        a = f("dh") * w1
        out["w_pre"] = torch.sum(f("dh") * nr, 0)
        if c["bias"]:
            out["b_pre"] = torch.sum(f("dh"), 0)
        d = d + rr * (a - nr * (torch.sum(a * nr, 1, keepdim=True) / D) - (torch.sum(a, 1, keepdim=True) / D if layer else 0))
    out["dx"] = 0.9 * d
    if c["gate"] != "none":
        t = 0.7 * d * oy
        out.update({"gate": t.sum(0)} if c["gate"] == "channel" else {"dgate": t})
    d = 0.7 * d * gate
    if c["post"]:
        a = d * w2
        out["w_post"] = torch.sum(d * ny, 0)
        if c["bias"]:
            out["b_post"] = torch.sum(d, 0)
        d = ry * (a - ny * (torch.sum(a * ny, 1, keepdim=True) / D) - (torch.sum(a, 1, keepdim=True) / D if layer else 0))
    out["dy"] = d
    return out


def _exact_route(c, s):
    l = s["logits"].double()
    T, E, k, G = c["T"], c["E"], c["k"], c["groups"]
    shut = l == -math.inf
    if c["score"] == "softmax":
        p = torch.softmax(torch.where(shut.all(1, keepdim=True), 0.0, l), 1) * ~shut
    else:
        p = 1 / (1 + torch.exp(-l))
    if c["dir"] == "fwd":
        rank = p + s["bias"].double() if c["bias"] else p if G > 1 else l
        rank = rank.masked_fill(shut, -1e30)
        if G > 1:      # out of the groups that are kept, one after the other
            g = rank.view(T, G, E // G)
            first = g.amax(2)
            if c["group_top"] == 2 and E // G > 1:
                rest = g.scatter(2, g.argmax(2, keepdim=True), -math.inf).amax(2)
                first = first + rest * (rest > -1e29)
            out = torch.ones(T, G, dtype=torch.bool, device=DEV)
            for _ in range(c["kept"]):
                out.scatter_(1, torch.where(out, first, -math.inf).argmax(1, keepdim=True), False)
            rank = rank.masked_fill(out.repeat_interleave(E // G, 1), -1e60)
        ids = []
        for _ in range(k):
            best = rank.amax(1, keepdim=True)
            i = torch.where(rank == best, torch.arange(E, device=DEV), E).amin(1, keepdim=True)
            ids.append(i)
            rank = rank.scatter(1, i, -math.inf)
        ids = torch.cat(ids, 1)
        w = p.gather(1, ids) * ~shut.gather(1, ids)
        if c["renorm"]:
            w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
        return [ids.int(), c["scale"] * w]
    ids = s["ids"].long()
    a = torch.zeros_like(l).scatter_(1, ids, s["dweights"].double()) * ~shut
    at = torch.zeros_like(l).scatter_(1, ids, 1.0) * ~shut
    grow = p * (1 - p) if c["score"] == "sigmoid" else p       # (softmax: its sum's part is put in below)
    if c["renorm"]:
        q = p * at / (p * at).sum(1, keepdim=True).clamp_min(1e-300)
        d = q * (a - (q * a).sum(1, keepdim=True))
        return c["scale"] * (d * (1 - p) if c["score"] == "sigmoid" else d)
    return c["scale"] * (grow * a if c["score"] == "sigmoid" else grow * (a - (p * a).sum(1, keepdim=True)))


def _exact_combine(c, s):
    yk = s["yk"].double().view(c["T"], c["k"], c["D"])
    if c["dir"] == "fwd":
        return torch.einsum("tk,tkd->td", s["weights"].double(), yk)
    dy = s["dy"].double()
    return [torch.einsum("tk,td->tkd", s["weights"].double(), dy).reshape(-1, c["D"]), torch.einsum("td,tkd->tk", dy, yk)]


def _exact_adamw(c, s):
    t, lr, byte = s["step"] + 1, 1e-3, c["state"] == "8bit"
    seed = (s["seed"] + 0x9E3779B9) & 0xFFFFFFFF
    m0, v0 = (_decode(s["m"], s["exps"][:, 0], TOP_M), _decode(s["v"], s["exps"][:, 1], TOP_V)) if byte else (s["m"].double(), s["v"].double())
    g = s["g"].double() * s["clip"].double()
    m, v = torch.lerp(g, m0, BETA1), torch.lerp(g.square(), v0, BETA2)
    p = (s["master"] if c["master"] else s["w"]).double()
    p = p - lr * s["wd"].double().expand(-1, BLOCK).reshape(-1) * p - lr * (m / (1 - BETA1 ** t)) / (torch.sqrt(v / (1 - BETA2 ** t)) + EPS)
    out = {"w": p}
    if c["master"]:
        out["master"] = p
    if c["dtype"] == "bf16" and not c["master"]:       # the two neighbours, and how far between them
        e = torch.frexp(p).exponent - 8
        out["w"] = torch.copysign(torch.floor(p.abs() * _two(-e) + _bits(seed, p.numel())[2] / 65536.0) * _two(e), p)
    if byte:
        rm, rv, _ = _bits(seed, p.numel())
        m, v = _exact_kept(m, TOP_M, rm), _exact_kept(v, TOP_V, rv)
    return {**out, "m": m, "v": v}


def _exact_kept(x, top, rnd):
    """what 8 bits keep of x: a multiple of an eighth of its binade, and below the last binade of that one's"""
    a = x.abs()
    binade = lambda t: torch.frexp(t.clamp_min(2.0 ** -126)).exponent - 1   # noqa: E731
    last = binade(a.view(-1, BLOCK).amax(1)) - (top - 1)
    e = torch.maximum(binade(a).view(-1, BLOCK), last[:, None]).view(-1) - 3
    kept = torch.floor(a * _two(-e) + rnd / 65536.0)
    if top == TOP_V:
        kept = torch.where(a > 0, kept.clamp_min(1), kept)
    return torch.copysign(kept * _two(e), x)
