"""What stands around a rotated unit in a training step: the router in front of an expert-partitioned layer, the
combination of a token's experts, the norms, gate and residual between units, and the AdamW step over the ring stores.

Checks of the tensors and marshalling only; the arithmetic is librtp.so's (include/rtp.h).  As with the layers, the
caller brings the outputs.  Every call runs on the caller's current stream, keeps nothing of its inputs and may be
captured into a graph (not an optimizer's step over layers: their rings refuse a stream that is being captured).  Tensors that come
from another stream are the caller's to order, and so are those that an object makes, on the stream it was made on.
"""
import ctypes as C

import torch

from . import binding as B

_RTP_DT = {torch.float32: B.RTP_F32, torch.bfloat16: B.RTP_BF16, torch.float16: B.RTP_F16}
_route_fwd, _route_bwd = B.lib.rtp_route_fwd, B.lib.rtp_route_bwd
_combine_fwd, _combine_bwd = B.lib.rtp_combine_fwd, B.lib.rtp_combine_bwd
_norm_fwd, _norm_bwd = B.lib.rtp_norm_fwd, B.lib.rtp_norm_bwd


def _rows(t, name, dtype, T, cols, dev):
    """Address and leading dimension of a [T, cols] matrix of `dtype` on `dev`, whose rows are contiguous."""
    try:
        if t.dtype is dtype and t.device == dev and t.shape == (T, cols):
            if t.is_contiguous():
                return t.data_ptr(), cols
            ld, step = t.stride()
            if T <= 1:
                ld = max(ld, cols)
            if ld >= cols and (step == 1 or cols == 1):
                return t.data_ptr(), ld
            raise ValueError(f"{name} must have contiguous rows that do not overlap")
    except AttributeError:       # no tensor
        pass
    raise ValueError(f"{name} must be a [{T}, {cols}] tensor of {dtype} on {dev}")


def _whole(t, name, dtype, shape, dev):
    """Address of a contiguous tensor."""
    try:
        if t.dtype is dtype and t.device == dev and t.shape == shape and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    raise ValueError(f"{name} must be a contiguous {list(shape)} tensor of {dtype} on {dev}")


def _gpu(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a tensor on the GPU")
    return t.device


def _float_type(t, name):
    code = _RTP_DT.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be float32, bfloat16 or float16")
    return code


# (what torch.cuda.current_device() and current_stream() look up, without the objects they make of it: 3 us a call)
_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _call(fn, where, dev, *args):
    """fn(*args, stream) on the caller's current stream of `dev`."""
    if _device() != dev.index:
        with torch.cuda.device(dev):
            status = fn(*args, _raw_stream(dev.index))
    else:
        status = fn(*args, _raw_stream(dev.index))
    if status:
        raise B.RtpError(status, where)


class RtpRouter:
    """Chooses `top_k` of `experts` experts for each token from its logits (rtp_route_fwd says how).  `bias`: fp32 [experts],
    added for the choice only; the caller moves it between steps."""

    def __init__(self, experts, top_k, score="softmax", renormalise=True, scale=1.0, groups=1, kept_groups=1, group_top=1, bias=None):
        if score not in ("softmax", "sigmoid"):
            raise ValueError("score is 'softmax' or 'sigmoid'")
        d = self.desc = B.rtp_route_desc()
        d.E, d.k, d.renormalise, d.scale = experts, top_k, int(bool(renormalise)), scale
        d.score = B.RTP_SCORE_SIGMOID if score == "sigmoid" else B.RTP_SCORE_SOFTMAX
        d.groups, d.kept_groups, d.group_top = groups, kept_groups, group_top
        self.bias = bias
        B.check(B.lib.rtp_route_fwd(C.byref(d), None, None, None, None, None), "rtp_route_fwd")   # T = 0: the checks alone

    def forward(self, logits, ids, weights):
        """logits [T, experts] -> ids int32 [T, top_k] (what RtpMoe takes as its route), weights fp32 [T, top_k]."""
        dev = _gpu(logits, "logits")
        d, logits_p = self._desc(logits, dev)
        shape = (d.T, d.k)
        ids_p, w_p = _whole(ids, "ids", torch.int32, shape, dev), _whole(weights, "weights", torch.float32, shape, dev)
        bias = None if self.bias is None else _whole(self.bias, "bias", torch.float32, (d.E,), dev)
        _call(_route_fwd, "rtp_route_fwd", dev, C.byref(d), logits_p, bias, ids_p, w_p)

    def backward(self, logits, ids, dweights, dlogits):
        """Gradient of the weights -> that of the logits (in the type of `dlogits`), for the ids of forward()."""
        dev = _gpu(logits, "logits")
        d, logits_p = self._desc(logits, dev)
        shape = (d.T, d.k)
        ids_p, dw_p = _whole(ids, "ids", torch.int32, shape, dev), _whole(dweights, "dweights", torch.float32, shape, dev)
        if not isinstance(dlogits, torch.Tensor):
            raise ValueError("dlogits must be a tensor")
        d.grad_dtype = _float_type(dlogits, "dlogits")
        dl_p, d.ld_grad = _rows(dlogits, "dlogits", dlogits.dtype, d.T, d.E, dev)
        _call(_route_bwd, "rtp_route_bwd", dev, C.byref(d), logits_p, ids_p, dw_p, dl_p)

    def _desc(self, logits, dev):
        d = B.rtp_route_desc.from_buffer_copy(self.desc)      # (two threads may share a router)
        if logits.dim() != 2:
            raise ValueError("logits must be [tokens, experts]")
        d.dtype, d.T = _float_type(logits, "logits"), logits.shape[0]
        p, d.ld = _rows(logits, "logits", logits.dtype, d.T, d.E, dev)
        return d, p


class RtpCombine:
    """Between tokens and their `top_k` slots (slot j of token t is row t * top_k + j)."""

    def __init__(self, top_k):
        if not 1 <= top_k <= B.RTP_COMBINE_MAX_TOP:
            raise ValueError(f"top_k is 1 to {B.RTP_COMBINE_MAX_TOP}")
        self.k = top_k

    def forward(self, Yk, weights, Y):
        """Y[t] = sum over a token's slots of weight * Yk (weights None: the plain sum, the gradient of expand())."""
        dev = _gpu(Y, "Y")
        T, D = self._tokens(Y, "Y")
        yk, ld_yk = _rows(Yk, "Yk", Y.dtype, T * self.k, D, dev)
        y, ld_y = _rows(Y, "Y", Y.dtype, T, D, dev)
        _call(_combine_fwd, "rtp_combine_fwd", dev, T, self.k, D, _float_type(Y, "Y"), yk, ld_yk, self._weights(weights, T, dev), y, ld_y)

    def backward(self, dY, Yk, weights, dYk, dweights=None):
        """dYk = weight * dY and, where asked for, dweights = <dY, Yk>.  (Yk may be None without dweights.)"""
        dev = _gpu(dY, "dY")
        T, D = self._tokens(dY, "dY")
        dy, ld_dy = _rows(dY, "dY", dY.dtype, T, D, dev)
        yk, ld_yk = (None, 0) if Yk is None else _rows(Yk, "Yk", dY.dtype, T * self.k, D, dev)
        dyk, ld_dyk = (None, 0) if dYk is None else _rows(dYk, "dYk", dY.dtype, T * self.k, D, dev)
        dw = None if dweights is None else _whole(dweights, "dweights", torch.float32, (T, self.k), dev)
        _call(_combine_bwd, "rtp_combine_bwd", dev, T, self.k, D, _float_type(dY, "dY"), dy, ld_dy, yk, ld_yk,
              self._weights(weights, T, dev), dyk, ld_dyk, dw)

    def expand(self, X, Xk):
        """Every token's row into its slots."""
        self.backward(X, None, None, Xk)

    def _weights(self, weights, T, dev):
        return None if weights is None else _whole(weights, "weights", torch.float32, (T, self.k), dev)

    @staticmethod
    def _tokens(t, name):
        if t.dim() != 2:
            raise ValueError(f"{name} must be [tokens, width]")
        return t.shape


_NONE = (None, 0)


class RtpNorm:
    """What lies between two units of a residual stream (rtp_norm_desc):

        r = res_scale * x + out_scale * gate * N_post(y);  h = N_pre(r)

    join: a unit's output y joins the stream; post: it is normalised first; pre: h is wanted.  Without join, h = N_pre(x).
    w_*, b_* and a channel gate are fp32 [D] parameters (None: 1, 0 and none); their gradients are fp32 and add up over
    backward passes, as those of the rotated units do, until zero_grads().  An element gate [T, D] goes into the calls."""

    _NAMES = ("w_post", "b_post", "w_pre", "b_pre", "gate")

    def __init__(self, D, kind="rms", eps=1e-5, join=True, post=False, pre=True, w_post=None, b_post=None, w_pre=None, b_pre=None, gate=None,
                 res_scale=1.0, out_scale=1.0, stream_dtype=torch.bfloat16, dtype=torch.bfloat16):
        if kind not in ("rms", "layer"):
            raise ValueError("kind is 'rms' or 'layer'")
        if (not post and (w_post is not None or b_post is not None)) or (not pre and (w_pre is not None or b_pre is not None)):
            raise ValueError("parameters of a norm that is left out")
        d = self.desc = B.rtp_norm_desc()
        self.dtype, self.stream_dtype = dtype, stream_dtype
        if dtype not in _RTP_DT or stream_dtype not in _RTP_DT:
            raise ValueError("types are float32, bfloat16 and float16")
        d.D, d.kind, d.eps = D, B.RTP_NORM_LAYER if kind == "layer" else B.RTP_NORM_RMS, eps
        d.parts = (B.RTP_NORM_JOIN if join else 0) | (B.RTP_NORM_POST if post else 0) | (B.RTP_NORM_PRE if pre else 0)
        d.stream_dtype, d.dtype, d.res_scale, d.out_scale = _RTP_DT[stream_dtype], _RTP_DT[dtype], res_scale, out_scale
        self.params = {n: t for n, t in zip(self._NAMES, (w_post, b_post, w_pre, b_pre, gate)) if t is not None}
        self.dev = None
        for n, t in self.params.items():
            self.dev = self.dev or _gpu(t, n)
            setattr(d, n + "_dev", _whole(t, n, torch.float32, (D,), self.dev))
        d.gate = B.RTP_GATE_NONE if gate is None else B.RTP_GATE_CHANNEL
        self.join, self.post, self.pre, self.D = join, post, pre, D
        self.grads = {n: torch.zeros_like(t) for n, t in self.params.items()}
        at = {n: t.data_ptr() for n, t in self.grads.items()}
        self._dparams, self._dgate = [at.get(n) for n in self._NAMES[:4]], at.get("gate")
        self._ws = (-1, 0)                                    # tokens, and the workspace they need
        B.check(B.lib.rtp_norm_fwd(C.byref(d), C.byref(B.rtp_norm_io()), None), "rtp_norm_fwd")     # T = 0: the checks alone

    def forward(self, x, y, r, h, stats, gate=None):
        """x, y -> r, h and stats (fp32 [T, 4], for backward).  y and r are None without join, h without pre."""
        dev = self._dev(x, "x")
        T = x.shape[0]
        d = self._desc(T, gate, dev)
        S, U, D = self.stream_dtype, self.dtype, self.D
        x_p, ld_x = _rows(x, "x", S, T, D, dev)
        y_p, ld_y = _rows(y, "y", U, T, D, dev) if self.join else _NONE
        r_p, ld_r = _rows(r, "r", S, T, D, dev) if self.join else _NONE
        h_p, ld_h = _rows(h, "h", U, T, D, dev) if self.pre else _NONE
        st_p = _whole(stats, "stats", torch.float32, (T, 4), dev) if self.pre or self.post else None
        _call(_norm_fwd, "rtp_norm_fwd", dev, C.byref(d), C.byref(B.rtp_norm_io(x_p, y_p, r_p, h_p, st_p, ld_x, ld_y, ld_r, ld_h)))

    def backward(self, r, y, dr, dh, dx, dy, stats, gate=None, dgate=None, accumulate=True):
        """dr (None: nothing follows), dh -> dx, dy, and the parameters' gradients, which it returns (the object's own fp32 tensors;
        accumulate=False overwrites them).  r is forward()'s, or x without join."""
        dev = self._dev(dx, "dx")
        T = dx.shape[0]
        d = self._desc(T, gate, dev)
        S, U, D = self.stream_dtype, self.dtype, self.D
        dx_p, ld_dx = _rows(dx, "dx", S, T, D, dev)
        dr_p, ld_dr = _rows(dr, "dr", S, T, D, dev) if dr is not None else _NONE
        r_p, ld_r = _rows(r, "r", S, T, D, dev) if self.pre else _NONE
        dh_p, ld_dh = _rows(dh, "dh", U, T, D, dev) if self.pre else _NONE
        dy_p, ld_dy = _rows(dy, "dy", U, T, D, dev) if self.join else _NONE
        y_p, ld_y = _rows(y, "y", U, T, D, dev) if self.post or d.gate != B.RTP_GATE_NONE else _NONE
        st_p = _whole(stats, "stats", torch.float32, (T, 4), dev) if self.pre or self.post else None
        dg_p, ld_dg = self._dgate, 0
        if dgate is not None:
            if gate is None:
                raise ValueError("dgate without an element gate")
            dg_p, ld_dg = _rows(dgate, "dgate", U, T, D, dev)
        ws, need = None, 0
        if self.grads:
            of, need = self._ws
            if of != T:
                need = B.lib.rtp_norm_ws_bytes(C.byref(d))
                self._ws = T, need
            # (a block of torch's allocator: ordered with this stream, and the graph's own while one is captured)
            ws = torch.empty(need, dtype=torch.uint8, device=dev)
        g = B.rtp_norm_grads(r_p, y_p, dr_p, dh_p, st_p, dx_p, dy_p, dg_p, *self._dparams, 1 if accumulate else 0, None if ws is None else ws.data_ptr(),
                             need, ld_r, ld_y, ld_dr, ld_dh, ld_dx, ld_dy, ld_dg)
        _call(_norm_bwd, "rtp_norm_bwd", dev, C.byref(d), C.byref(g))
        return self.grads

    def zero_grads(self):
        for t in self.grads.values():
            t.zero_()

    def _dev(self, t, name):
        dev = _gpu(t, name)
        if self.dev is not None and dev != self.dev:
            raise ValueError(f"{name} is on {dev}, the parameters on {self.dev}")
        if t.dim() != 2:
            raise ValueError(f"{name} must be [tokens, {self.D}]")
        return dev

    def _desc(self, T, gate, dev):
        d = B.rtp_norm_desc.from_buffer_copy(self.desc)       # (two threads may share a norm)
        d.T = T
        if gate is not None:
            if d.gate != B.RTP_GATE_NONE:
                raise ValueError("a channel gate and an element gate")
            d.gate = B.RTP_GATE_ELEMENT
            d.gate_dev, d.ld_gate = _rows(gate, "gate", self.dtype, T, self.D, dev)
        return d


class RtpAdamW:
    """AdamW over many tensors as one launch (rtp_adamw_step).

    tensors: dicts of `param` (fp32, bf16 or fp16), `grad` (fp32), and optionally `master` (fp32, of a 16-bit parameter) and
    `weight_decay` (0), contiguous, of one size.  state: 'f32' or '8bit' moments.  `moments`: (m, v, exps) to go on from,
    flat as rtp_adamw_desc lays them out (exps None for 'f32'); fresh ones are zeros.  16-bit parameters without a master
    copy and 8-bit moments are rounded at random, from the seed of the step."""

    def __init__(self, tensors, state="f32", moments=None):
        if state not in ("f32", "8bit"):
            raise ValueError("state is 'f32' or '8bit'")
        self.handle, self.layers, self.state = C.c_void_p(), [], state
        self._keep = [dict(t) for t in tensors]
        if not self._keep:
            raise ValueError("no tensors")
        arr = (B.rtp_adamw_tensor * len(self._keep))()
        self.dev = _gpu(self._keep[0].get("param"), "param")
        for e, t in zip(arr, self._keep):
            p, g, m = t["param"], t["grad"], t.get("master")
            e.dtype, e.numel = _float_type(p, "param"), p.numel()
            e.param_dev = _whole(p, "param", p.dtype, p.shape, self.dev)
            e.grad_dev = _whole(g, "grad", torch.float32, p.shape, self.dev)
            if m is not None:
                e.master_dev = _whole(m, "master", torch.float32, p.shape, self.dev)
            e.weight_decay = t.get("weight_decay", 0.0)
        self.blocks = B.lib.rtp_adamw_blocks(arr, len(arr))
        if self.blocks < 0:
            raise ValueError("an empty tensor, or too many")
        n, byte = self.blocks * B.RTP_ADAMW_BLOCK, state == "8bit"
        dt = torch.uint8 if byte else torch.float32
        if moments is None:
            moments = (torch.zeros(n, dtype=dt, device=self.dev), torch.zeros(n, dtype=dt, device=self.dev),
                       torch.zeros(self.blocks, 2, dtype=torch.uint8, device=self.dev) if byte else None)
        self.m, self.v, self.exps = moments
        self.table = torch.empty(B.lib.rtp_adamw_table_bytes(arr, len(arr)), dtype=torch.uint8, device=self.dev)
        d = B.rtp_adamw_desc()
        d.tensors, d.count, d.moments = arr, len(arr), B.RTP_MOMENTS_8BIT if byte else B.RTP_MOMENTS_F32
        d.m_dev, d.v_dev = _whole(self.m, "m", dt, (n,), self.dev), _whole(self.v, "v", dt, (n,), self.dev)
        if byte:
            d.exps_dev = _whole(self.exps, "exps", torch.uint8, (self.blocks, 2), self.dev)
        d.table_dev = self.table.data_ptr()
        with torch.cuda.device(self.dev):
            d.stream = torch.cuda.current_stream(self.dev).cuda_stream
            B.check(B.lib.rtp_adamw_create(C.byref(self.handle), C.byref(d)), "rtp_adamw_create")

    @classmethod
    def for_layers(cls, layers, state="f32", master=False, weight_decay=0.0, more=()):
        """Over the ring stores of rotated layers (RtpLinear, RtpMlp, RtpMoe), every slot a tensor, and `more` tensors.
        step() then brings each layer's shards home first and clears their gradients afterwards.  `weight_decay` is of whole
        slots, a layer's biases among them."""
        tensors = list(more)
        for layer in layers:
            dt = {v: k for k, v in _RTP_DT.items()}[layer.dtype]
            for w, g in zip(layer.home_w, layer.home_g):
                w, g = w.view(dt), g.view(torch.float32)
                n = min(w.numel(), g.numel())                 # (a slot's end is filled up to 16 bytes)
                t = dict(param=w[:n], grad=g[:n], weight_decay=weight_decay)
                if master and dt != torch.float32:
                    t["master"] = w[:n].float()
                tensors.append(t)
        opt = cls(tensors, state)
        opt.layers = list(layers)
        return opt

    def step(self, lr, step, betas=(0.9, 0.999), eps=1e-8, seed=None, grad_scale=None, scalars=None):
        """step: 1 for the first.  seed: 32 bits, another one every step (None: made from `step`).  grad_scale: a device scalar
        the gradients are multiplied by; not finite, the step changes nothing.  scalars: a device tensor with what
        scalars_of() gives, read when the step runs (for steps in a graph); lr, step, betas, eps and seed are not looked at then."""
        h, sc = None, None
        if scalars is None:
            h = C.byref(self._hyper(lr, step, betas, eps, seed))
        else:
            sc = _whole(scalars, "scalars", torch.uint8, (C.sizeof(B.rtp_adamw_scalars),), self.dev)
        if grad_scale is not None and not (isinstance(grad_scale, torch.Tensor) and grad_scale.numel() == 1):
            raise ValueError("grad_scale must be a tensor of one value")
        gs = None if grad_scale is None else _whole(grad_scale.reshape(1), "grad_scale", torch.float32, (1,), self.dev)
        if self.layers:         # (what the step itself would refuse, before the layers' shards have gone home for it)
            if not self.handle:
                B.check(B.lib.rtp_adamw_step(None, h, sc, gs, None), "rtp_adamw_step")
            if h is not None:
                B.check(B.lib.rtp_adamw_scalars_of(h, C.byref(B.rtp_adamw_scalars())), "rtp_adamw_step")
            elif sc % 16:
                raise ValueError("scalars must be at a multiple of 16 bytes")
        for layer in self.layers:
            layer._enter()
            B.check(B.lib.rtp_ring_flush(layer.ring_handle()), "rtp_ring_flush")
            layer._leave()
        _call(B.lib.rtp_adamw_step, "rtp_adamw_step", self.dev, self.handle, h, sc, gs)
        for layer in self.layers:
            layer._enter()
            B.check(B.lib.rtp_ring_zero_grads(layer.ring_handle()), "rtp_ring_zero_grads")
            layer._leave()

    @staticmethod
    def _hyper(lr, step, betas, eps, seed):
        h = B.rtp_adamw_hyper()
        h.lr, h.step, h.eps = lr, step, eps
        h.beta1, h.beta2 = betas
        h.seed = (step * 0x9E3779B9 if seed is None else seed) & 0xFFFFFFFF
        return h

    @classmethod
    def scalars_of(cls, lr, step, betas=(0.9, 0.999), eps=1e-8, seed=None):
        """One step's values as a host tensor, for copying to the device tensor a captured step reads."""
        out = B.rtp_adamw_scalars()
        B.check(B.lib.rtp_adamw_scalars_of(C.byref(cls._hyper(lr, step, betas, eps, seed)), C.byref(out)), "rtp_adamw_scalars_of")
        return torch.frombuffer(bytearray(bytes(out)), dtype=torch.uint8)

    def moments(self, dtype=None):
        """(m, v) as numbers, flat in blocks; fp32, or bf16 (8-bit moments' default, which holds them exactly)."""
        dtype = dtype or (torch.bfloat16 if self.state == "8bit" else torch.float32)
        if dtype not in _RTP_DT:
            raise ValueError("moments are handed out in float32 or bfloat16")
        m = torch.empty(self.blocks * B.RTP_ADAMW_BLOCK, dtype=dtype, device=self.dev)
        v = torch.empty_like(m)
        _call(B.lib.rtp_adamw_moments, "rtp_adamw_moments", self.dev, self.handle, _RTP_DT[dtype], m.data_ptr(), v.data_ptr())
        return m, v

    def close(self):
        if self.handle:
            B.check(B.lib.rtp_adamw_destroy(self.handle), "rtp_adamw_destroy")
            self.handle = C.c_void_p()
