"""Drop-in layers whose backward yields the clipped, noised gradient of their parameters (the paper's delivery
vehicle, Section 4.2: operators with trainable parameters are wrapped in an autograd function).

Only glue lives here.  The weight gradient - the whole path of Algorithm 1 - comes from the HIP library
through flashdp_block_dp_grad.  A linear layer without an epilogue leaves its forward product Y = X W^T to torch.matmul; with a bias, an
activation, a residual or 8-bit checkpoints the library forms it (flashdp_linear_forward) and its
backward (flashdp_activation_dp_grad).  The input gradient dX = dZ W is a plain GEMM left to torch.matmul.  Layer
normalisation is the library's in both directions.

The loss must be a SUM over samples (not a mean), so that dY[i] is sample i's own output gradient; the
batch dimension is the first one and everything between it and the feature dimension counts as tokens.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as F


class deferred_weight_grads:
    """Context manager: DPLinear backward passes inside it only record (X, dY) of their layer; on exit all
    recorded layers go to the library in ONE flashdp_block_dp_grad call per (device, B, T, dtype) group, so that the
    per-block schedule applies (the aggregation of one layer running beside the contraction of the next)
    instead of one isolated call per layer (layers with 8-bit checkpoints go together too, but are computed one
    after the other: each keeps a checkpoint of its own, and unpacks it in front of its contraction).  The weights' .grad fields are filled (or added to) on exit.  The
    price is that X and dY of every recorded layer stay alive until then; one that has been written in place by then is an
    error, as it is for what autograd saves."""

    _active = None

    def __init__(self, schedule="auto"):
        self.schedule = schedule
        self.pending = []

    def __enter__(self):
        if deferred_weight_grads._active is not None:
            raise RuntimeError("deferred_weight_grads does not nest")
        deferred_weight_grads._active = self
        return self

    def __exit__(self, exc_type, exc, tb):
        deferred_weight_grads._active = None
        try:
            if exc_type is None:
                self.flush()
        finally:
            self.pending = []
        return False

    def flush(self):
        groups = {}
        for rec in self.pending:
            if _versions(rec["X"], rec["dY"]) != rec["versions"]:
                raise RuntimeError("the input or the output gradient of a layer was modified in place before the deferred weight gradients were computed")
            _check_capture(rec["module"], rec["sigma"], rec["add_noise"])
        for rec in self.pending:
            groups.setdefault((rec["X"].device, rec["B"], rec["T"], rec["dY"].dtype, rec["packed"]), []).append(rec)
        for (device, B, T, _, packed), recs in groups.items():
            with torch.cuda.device(device):
                self._flush_group(recs, B, T, packed)
        self.pending = []

    def _flush_group(self, recs, B, T, packed):
        grad = _grad_call(packed)
        layers = []
        for r in recs:
            r["out"] = torch.empty(r["weight"].shape, dtype=torch.float32, device=r["X"].device)
            layers.append(dict(X=r["X"], dY=r["dY"], d_in=r["weight"].shape[1], d_out=r["weight"].shape[0], C=r["C"],
                               sigma=r["sigma"], seed=r["seed"], layer=r["layer"], out_grad=r["out"], out_norms=r["norms"]))
        # layers of one group share the noise flag only if they agree; otherwise one call per flag value
        for flag in sorted({r["add_noise"] for r in recs}, reverse=True):
            sub = [L for L, r in zip(layers, recs) if r["add_noise"] == flag]
            grad(sub, B, T, F.dtype_code(recs[0]["dY"]), self.schedule, accumulate=False, add_noise=flag)
        for r in recs:
            if r["module"] is not None and r["module"].keep_fp32_grad:
                m = r["module"]
                m.grad_fp32 = r["out"].clone() if m.grad_fp32 is None else m.grad_fp32 + r["out"]
            g = r["out"].to(r["weight"].dtype)
            r["weight"].grad = g if r["weight"].grad is None else r["weight"].grad + g


def _versions(*tensors):
    """How often their memory was written in place (not counted for tensors made in inference mode)."""
    return tuple(0 if t.is_inference() else t._version for t in tensors)


def _check_capture(module, sigma, add_noise):
    """What a graph keeps of a call is the seed's value, so every replay adds the same noise.  A module that counts its steps by itself has
    promised another field for each of them, and does not have its noise captured."""
    if module is not None and module.auto_step and add_noise and sigma > 0 and torch.cuda.is_current_stream_capturing():
        raise RuntimeError("a graph's replays would repeat the noise of its capture: capture with add_noise = False (or sigma = 0) and add the noise outside "
                           "the graph, or set auto_step = False, which leaves steps and seeds to the caller")


def _grad_call(packed):
    """The block call for activations as they are, or for 8-bit checkpoints of them.  Both take the library's workspace, or, while a graph is
    being captured, one of torch's: the graph keeps its memory, where the library's would be freed by a later call that makes it grow."""
    grad, size = ((F.flashdp_block_dp_grad_checkpoint8, F.flashdp_workspace_bytes_checkpoint8) if packed
                  else (F.flashdp_block_dp_grad_micro, F.flashdp_workspace_bytes))
    if not torch.cuda.is_current_stream_capturing():
        return grad

    def call(layers, B, T, dtype, schedule, **kw):
        room = schedule
        if F.schedule_code(schedule) == F.SCHEDULE_AUTO:      # rows without a sequence park nothing; two layers or more can take turns in two slots
            room = "twopass" if T == 1 and B > 1 else "overlap" if len(layers) > 1 else "scratch"
        grad(layers, B, T, dtype, schedule, _workspace(size(layers, B, T, dtype, room), layers[0]["X"].device), **kw)

    return call


def _weight_grad(X, packed, dY, B, T, weight, C, sigma, seed, layer, schedule, norms, add_noise, module, incoming):
    """The weight's gradient, now or - inside deferred_weight_grads, where None is returned - in the block call at its end.  X is the
    activation [B, T, d_in], or with `packed` its 8-bit checkpoint.  incoming: the tensor that autograd handed to the backward pass.  dY may be
    another view of its memory, which autograd does not count: it would give an incoming gradient that nobody else holds to a leaf as its .grad
    and add the next pass's to it in place.  So the record holds that very tensor as well."""
    pending = deferred_weight_grads._active
    if pending is not None:   # hand the layer to the per-block call made when the context exits
        pending.pending.append(dict(X=X, packed=packed, dY=dY, incoming=incoming, versions=_versions(X, dY), B=B, T=T, weight=weight, C=C, sigma=sigma,
                                    seed=seed, layer=layer, norms=norms, add_noise=add_noise, module=module))
        return None
    _check_capture(module, sigma, add_noise)
    d_out, d_in = weight.shape
    grad_w = torch.empty((d_out, d_in), dtype=torch.float32, device=dY.device)
    L = [dict(X=X, dY=dY, d_in=d_in, d_out=d_out, C=C, sigma=sigma, seed=seed, layer=layer, out_grad=grad_w, out_norms=norms)]
    _grad_call(packed)(L, B, T, F.dtype_code(dY), schedule, accumulate=False, add_noise=add_noise)
    if module is not None and module.keep_fp32_grad:
        module.grad_fp32 = grad_w.clone() if module.grad_fp32 is None else module.grad_fp32 + grad_w
    return grad_w.to(weight.dtype)


class _DPLinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, C, sigma, seed, layer, schedule, norms_out, add_noise, module):
        ctx.save_for_backward(x, weight)
        ctx.cfg = (float(C), float(sigma), int(seed), int(layer), schedule, norms_out, bool(add_noise), module)
        return torch.matmul(x, weight.t())

    @staticmethod
    def backward(ctx, dy):
        x, weight = ctx.saved_tensors
        C, sigma, seed, layer, schedule, norms_out, add_noise, module = ctx.cfg
        nothing = (None,) * 8
        d_out, d_in = weight.shape
        B = x.shape[0]
        xs = x.reshape(B, -1, d_in).contiguous()
        dys = dy.reshape(B, -1, d_out).contiguous()
        T = xs.shape[1]
        if xs.dtype != dys.dtype:
            dys = dys.to(xs.dtype)
        norms = norms_out if norms_out is not None else torch.empty((B,), dtype=torch.float32, device=x.device)
        grad_x = torch.matmul(dy, weight) if ctx.needs_input_grad[0] else None
        grad_w = _weight_grad(xs, False, dys, B, T, weight, C, sigma, seed, layer, schedule, norms, add_noise, module, dy)
        return (grad_x, grad_w) + nothing


def _dense(t):
    """t with rows one after the other from a 16-byte boundary on, as the library wants it: t itself, or a copy."""
    t = t.detach().contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _workspace(nbytes, device):
    """Room for one call, from torch's allocator: ordered by the stream, and a captured graph keeps its own."""
    return torch.empty((max(nbytes, 16),), dtype=torch.uint8, device=device)


class _DPLinearEpilogueFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, module, seed, norms, bias_norms, grad_mode):
        d_out, d_in = weight.shape
        if x.dim() < 2 or x.shape[-1] != d_in:
            raise TypeError(f"the input is [samples, ..., {d_in}], not {tuple(x.shape)}")
        if x.dtype != weight.dtype or (residual is not None and (residual.dtype != x.dtype or residual.shape != (*x.shape[:-1], d_out))):
            raise TypeError("input, weight and residual need one dtype, and the residual the output's shape")
        xs = _dense(x)
        rows, code = xs.numel() // d_in, F.dtype_code(xs)
        eight, act = module.checkpoint == "8bit", module.activation
        with torch.cuda.device(x.device):
            y = torch.empty((*x.shape[:-1], d_out), dtype=x.dtype, device=x.device)
            train = grad_mode and any(ctx.needs_input_grad)
            z = None
            if train and act is not None:
                z = (torch.empty((F.flashdp_checkpoint8_bytes(rows, d_out),), dtype=torch.uint8, device=x.device) if eight
                     else torch.empty_like(y))
            F.flashdp_linear_forward(xs, _dense(weight), None if bias is None else _dense(bias),
                                     None if residual is None else _dense(residual), rows, d_in, d_out, code, act, y, z, eight and z is not None)
            kept = None
            if train and ctx.needs_input_grad[1]:
                kept = xs
                if eight:
                    kept = torch.empty((F.flashdp_checkpoint8_bytes(rows, d_in),), dtype=torch.uint8, device=x.device)
                    F.flashdp_checkpoint8_pack(xs, rows, d_in, code, kept)
        ctx.save_for_backward(kept, z, weight)
        ctx.cfg = (module, seed, norms, bias_norms, x.shape[0], rows // x.shape[0], eight, act, module.C, module.bias_C, module.sigma,
                   module.layer, module.schedule, module.add_noise)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        kept, z, weight = ctx.saved_tensors
        module, seed, norms, bias_norms, B, T, eight, act, C, bias_C, sigma, layer, schedule, add_noise = ctx.cfg
        need_x, need_w, need_b, need_r = ctx.needs_input_grad[:4]
        d_out, d_in = weight.shape
        grad_x = grad_w = grad_b = None
        if need_b:
            _check_capture(module, sigma, add_noise)
        with torch.cuda.device(dy.device):
            dys = _dense(dy.to(weight.dtype))
            dz = dys
            if act is not None or need_b:
                if act is not None:
                    dz = torch.empty_like(dys)
                code = F.dtype_code(dys)
                gb = torch.empty((d_out,), dtype=torch.float32, device=dy.device) if need_b else None
                ws = _workspace(F.flashdp_activation_workspace_bytes(B, T, d_out, code), dy.device) if need_b else None
                F.flashdp_activation_dp_grad(dys, z, eight and z is not None, B, T, d_out, code, act, bias_C, sigma, seed, layer,
                                             dz if act is not None else None, gb, bias_norms if need_b else None, ws, add_noise=add_noise)
                if need_b:
                    if module.keep_fp32_grad:
                        module.bias_grad_fp32 = gb.clone() if module.bias_grad_fp32 is None else module.bias_grad_fp32 + gb
                    grad_b = gb.to(weight.dtype)
            if need_x:
                grad_x = torch.matmul(dz, weight)
            if need_w:
                grad_w = _weight_grad(kept if eight else kept.reshape(B, T, d_in), eight, dz.reshape(B, T, d_out), B, T, weight, float(C), float(sigma),
                                      seed, layer, schedule, norms, add_noise, module, dy)
        return grad_x, grad_w, grad_b, dy if need_r else None, None, None, None, None, None


class _DPModule(torch.nn.Module):
    """What layers with a DP gradient share: threshold, noise multiplier, and the bookkeeping of seeds and steps.

    Noise and steps.  The Philox field is keyed by (seed, step, layer): `step` is folded into the seed, and with
    auto_step (the default) it advances by itself at every forward pass whose backward adds noise, so that two
    optimizer steps never receive the same field - the Gaussian mechanism of Algorithm 1 would be void otherwise
    (the difference of two updates would be noise-free).  last_seed is the seed the last forward pass used.
    A backward pass captured into a graph keeps its seed: every replay adds the same field.  With auto_step a backward pass that
    adds noise therefore refuses to be captured; without, the noise is that of `step` as the caller has set it, and a graph's is that of
    the capture for good - replays are steps of one mechanism only where the caller adds fresh noise outside the graph.
    Gradient accumulation over micro-batches (Appendix D.1): set add_noise = False for all micro-batches of a step but
    the last; every micro-batch is clipped per sample, torch sums the clipped sums in .grad, and the noise goes
    in once, with the last micro-batch (the step then advances once, too).
    A parameter's .grad has the parameter's dtype; with keep_fp32_grad the unrounded fp32 sum is kept as well
    (the caller clears it with zero_fp32_grad())."""

    def __init__(self, C, sigma, seed, layer, auto_step, keep_fp32_grad):
        super().__init__()
        self.C, self.sigma, self.seed, self.layer = C, sigma, seed, layer
        self.step = 0
        self.auto_step = auto_step
        self.add_noise = True
        self.keep_fp32_grad = keep_fp32_grad
        self.grad_fp32 = None
        self.last_norms = None
        self.last_seed = None

    def noise_seed(self) -> int:
        return (self.seed + (self.step << 32)) & 0xFFFFFFFFFFFFFFFF

    def zero_fp32_grad(self):
        self.grad_fp32 = None

    def _advance(self):
        if self.auto_step and self.add_noise and torch.is_grad_enabled():
            self.step += 1


class DPLinear(_DPModule):
    """y = act(x W^T + bias) + residual.  After backward(), weight.grad holds (torch adds across backward calls)
    sum_i clip(G_i) + sigma*C*z, and last_norms the per-sample norms; see _DPModule for noise, steps and keep_fp32_grad.

    bias: a bias whose gradient is clipped and noised by itself (threshold bias_C, by default C; norms in last_bias_norms, the fp32 sum in
    bias_grad_fp32), which makes sqrt(C^2 + bias_C^2) the layer's sensitivity.  activation: None, "relu", "gelu", "gelu_tanh" or
    "silu".  checkpoint: None keeps the input and the sum in front of the activation as they are between forward and backward pass,
    "8bit" keeps both in 8 bits (flashdp_checkpoint8_pack), 33/32 bytes an element instead of 2 or 4; the gradients are those at the values that
    were kept, clipped for what they are.  Every layer keeps a checkpoint of its own: layers that share an input (q, k, v; gate and up) share one tensor
    without checkpoints, so three of them in 16-bit types keep 3.1 bytes an element with checkpoints and 2 without.

    The weight gradient takes the library's workspace, one per device: backward passes of one device run on one stream."""

    def __init__(self, d_in: int, d_out: int, C: float = 1.0, sigma: float = 1.0, seed: int = 0, layer: int = 0,
                 schedule="auto", dtype=torch.bfloat16, device="cuda", auto_step: bool = True, keep_fp32_grad: bool = False,
                 bias: bool = False, activation=None, checkpoint=None, bias_C=None):
        super().__init__(C, sigma, seed, layer, auto_step, keep_fp32_grad)
        if activation == "none":
            activation = None
        F.activation_code(activation)
        if checkpoint not in (None, "8bit"):
            raise ValueError(f"checkpoint {checkpoint!r}: None or '8bit'")
        self.weight = torch.nn.Parameter(torch.empty(d_out, d_in, dtype=dtype, device=device))
        torch.nn.init.normal_(self.weight, std=d_in ** -0.5)
        self.bias = torch.nn.Parameter(torch.zeros(d_out, dtype=dtype, device=device)) if bias else None
        self.schedule, self.activation, self.checkpoint = schedule, activation, checkpoint
        self.bias_C = C if bias_C is None else bias_C
        self.last_bias_norms = None
        self.bias_grad_fp32 = None

    def zero_fp32_grad(self):
        super().zero_fp32_grad()
        self.bias_grad_fp32 = None

    def forward(self, x, residual=None):
        self.last_norms = torch.empty((x.shape[0],), dtype=torch.float32, device=x.device)
        self.last_seed = self.noise_seed()
        if self.bias is None and self.activation is None and self.checkpoint is None and residual is None:
            y = _DPLinearFn.apply(x, self.weight, self.C, self.sigma, self.last_seed, self.layer, self.schedule,
                                  self.last_norms, self.add_noise, self)
        else:
            self.last_bias_norms = None if self.bias is None else torch.empty_like(self.last_norms)
            y = _DPLinearEpilogueFn.apply(x, self.weight, self.bias, residual, self, self.last_seed, self.last_norms, self.last_bias_norms,
                                          torch.is_grad_enabled())
        self._advance()
        return y


class _DPLayerNormFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, module, seed, norms):
        if x.dim() < 2 or x.dtype != weight.dtype or x.shape[-1] != weight.shape[0]:
            raise TypeError("input and weight need one dtype, and the input is [samples, ..., the weight's size]")
        d = weight.shape[0]
        xs = _dense(x)
        rows, code = xs.numel() // d, F.dtype_code(xs)
        with torch.cuda.device(x.device):
            y = torch.empty_like(xs)
            mean = torch.empty((rows,), dtype=torch.float32, device=x.device)
            rstd = torch.empty_like(mean)
            F.flashdp_layernorm_forward(xs, _dense(weight), None if bias is None else _dense(bias), rows, d, code, module.eps, y, mean, rstd)
        ctx.save_for_backward(xs, weight, mean, rstd)
        ctx.cfg = (module, seed, norms, x.shape[0], rows // x.shape[0], bias is not None, module.C, module.sigma, module.layer, module.add_noise)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        xs, weight, mean, rstd = ctx.saved_tensors
        module, seed, norms, B, T, has_bias, C, sigma, layer, add_noise = ctx.cfg
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        d, code = weight.shape[0], F.dtype_code(xs)
        with torch.cuda.device(dy.device):
            dys = _dense(dy.to(xs.dtype))
            dx = torch.empty_like(xs) if need_x else None
            # weight and bias are one vector with one norm, whichever of them is wanted
            need_g = need_w or need_b
            if need_g:
                _check_capture(module, sigma, add_noise)
            g = torch.empty((2 if has_bias else 1, d), dtype=torch.float32, device=dy.device) if need_g else None
            ws = _workspace(F.flashdp_layernorm_workspace_bytes(B, T, d, code, has_bias), dy.device) if need_g else None
            if need_x or need_g:
                F.flashdp_layernorm_dp_grad(xs, dys, _dense(weight), mean, rstd, B, T, d, code, C, sigma, seed, layer, dx, g, norms if need_g else None,
                                            has_bias, ws, add_noise=add_noise)
            if need_g and module.keep_fp32_grad:
                module.grad_fp32 = g.clone() if module.grad_fp32 is None else module.grad_fp32 + g
        return dx, g[0].to(weight.dtype) if need_w else None, g[1].to(weight.dtype) if need_b else None, None, None, None


class DPLayerNorm(_DPModule):
    """Layer normalisation over the last dimension whose weight and bias get the clipped, noised gradient of Algorithm 1, as one vector with
    one norm per sample (last_norms); see _DPModule for noise, steps and keep_fp32_grad (grad_fp32 is [2, d], weight first).  Samples
    are the first dimension, as in DPLinear."""

    def __init__(self, d: int, C: float = 1.0, sigma: float = 1.0, seed: int = 0, layer: int = 0, eps: float = 1e-5, bias: bool = True,
                 dtype=torch.bfloat16, device="cuda", auto_step: bool = True, keep_fp32_grad: bool = False):
        super().__init__(C, sigma, seed, layer, auto_step, keep_fp32_grad)
        self.eps = eps
        self.weight = torch.nn.Parameter(torch.ones(d, dtype=dtype, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(d, dtype=dtype, device=device)) if bias else None

    def forward(self, x):
        self.last_norms = torch.empty((x.shape[0],), dtype=torch.float32, device=x.device)
        self.last_seed = self.noise_seed()
        y = _DPLayerNormFn.apply(x, self.weight, self.bias, self, self.last_seed, self.last_norms)
        self._advance()
        return y
