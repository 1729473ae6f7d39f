"""`torch.autograd.Function` wrappers: the paper's YN post-process in PyTorch terms
(Section IV, component C: the saved tensor of the node becomes the FAD result, and its
backward function becomes a direct multiplication).  The wrappers only allocate tensors
and call the CUDA library.
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import binding as nfad
from . import block
from . import sequence


class NestedActivation(torch.autograd.Function):
    """y = f(x) with f'(x) as the only saved tensor; backward = grad_out * f'(x)."""

    @staticmethod
    def forward(ctx, x: torch.Tensor, kind: str):
        xc = x.contiguous()
        y = torch.empty_like(xc)
        d = torch.empty_like(xc)
        nfad.nfad_act_forward(kind, xc.view(-1), y.view(-1), d.view(-1))
        ctx.save_for_backward(d)
        ctx.kind = kind
        return y

    @staticmethod
    def backward(ctx, grad_out: torch.Tensor):
        (d,) = ctx.saved_tensors
        g = grad_out.contiguous()
        gin = torch.empty_like(g)
        nfad.nfad_act_backward(ctx.kind, g.view(-1), d.view(-1), gin.view(-1))
        return gin, None


class NestedBiasActivation(torch.autograd.Function):
    """y = f(x + bias) for x of shape [..., cols] and bias of shape [cols]: f'(x + bias) is the only saved tensor;
    backward gives grad_x = grad_out * f' and grad_bias = its column sums, from one kernel."""

    @staticmethod
    def forward(ctx, x: torch.Tensor, bias: torch.Tensor, kind: str):
        xc, bc = x.contiguous(), bias.contiguous()
        y = torch.empty_like(xc)
        d = torch.empty_like(xc)
        nfad.nfad_bias_act_forward(kind, xc.view(-1), bc, y.view(-1), d.view(-1))
        ctx.save_for_backward(d)
        ctx.kind, ctx.cols, ctx.bias_dtype = kind, bc.numel(), bias.dtype
        return y

    @staticmethod
    def backward(ctx, grad_out: torch.Tensor):
        (d,) = ctx.saved_tensors
        g = grad_out.contiguous()
        gin = torch.empty_like(g)
        gb = torch.empty(ctx.cols, dtype=torch.float32, device=g.device)
        nbytes = nfad.nfad_bias_act_backward_scratch_bytes(g.dtype, g.numel() // ctx.cols, ctx.cols, g.device)
        scratch = torch.empty(nbytes, dtype=torch.uint8, device=g.device) if nbytes else None
        nfad.nfad_bias_act_backward(ctx.kind, g.view(-1), d.view(-1), gin.view(-1), gb, scratch)
        return gin, gb.to(ctx.bias_dtype), None


class ConventionalActivation(torch.autograd.Function):
    """The comparator that saves x and re-derives f'(x) in one fused backward kernel."""

    @staticmethod
    def forward(ctx, x: torch.Tensor, kind: str):
        xc = x.contiguous()
        y = torch.empty_like(xc)
        nfad.nfad_act_forward_infer(kind, xc.view(-1), y.view(-1))
        ctx.save_for_backward(xc)
        ctx.kind = kind
        return y

    @staticmethod
    def backward(ctx, grad_out: torch.Tensor):
        (x,) = ctx.saved_tensors
        g = grad_out.contiguous()
        gin = torch.empty_like(g)
        nfad.nfad_cmp_conv_backward(ctx.kind, g.view(-1), x.view(-1), gin.view(-1))
        return gin, None


class FadSequence(torch.autograd.Function):
    """A run-time FAD sequence with M results: saves one derivative tensor per result."""

    @staticmethod
    def forward(ctx, x: torch.Tensor, prog: sequence.FadProgram):
        xc = x.contiguous()
        ys, ds = sequence.run_fused(prog, xc.view(-1))
        ctx.save_for_backward(*ds)
        ctx.shape = xc.shape
        return tuple(y.view(xc.shape) for y in ys)

    @staticmethod
    def backward(ctx, *grad_outs):
        ds = ctx.saved_tensors
        gs = [g.contiguous().view(-1) for g in grad_outs]
        return sequence.backward_fused(gs, list(ds)).view(ctx.shape), None


class BlockNormFunction(torch.autograd.Function):
    """(s, h) of the norms around a block; saved: u, s, four statistics a row, and the parameters."""

    @staticmethod
    def forward(ctx, u, r, post_gain, post_bias, gate, pre_gain, pre_bias, post, pre, residual_scale, eps):
        given = dict(post_gain=post_gain, post_bias=post_bias, gate=gate, pre_gain=pre_gain, pre_bias=pre_bias)
        given = {k: t.contiguous() for k, t in given.items() if t is not None}
        settings = dict(post=post, pre=pre, residual_scale=residual_scale, eps=eps)
        norm = block.BlockNorm(**given, **settings)
        uc, rc = u.contiguous(), None if r is None else r.contiguous()
        s = torch.empty_like(uc)
        h = torch.empty_like(uc) if norm.pre else None
        stats = torch.empty(uc.numel() // max(1, uc.shape[-1]), 4, device=uc.device)
        block.nfad_block_norm_forward(norm, uc, rc, s, h, stats)
        ctx.save_for_backward(uc, s, stats, *given.values())
        ctx.set_materialize_grads(False)             # a result that nothing used costs no read of zeros
        ctx.names, ctx.settings, ctx.r_shape = list(given), settings, None if r is None else r.shape
        if h is None:
            h = s.new_empty(0)
            ctx.mark_non_differentiable(h)
        return s, h

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_s, grad_h):
        u, s, stats, *given = ctx.saved_tensors
        norm = block.BlockNorm(**dict(zip(ctx.names, given)), **ctx.settings)
        if norm.pre and grad_h is None or not norm.pre and grad_s is None:
            zeros = torch.zeros_like(s)
            grad_h, grad_s = (zeros, grad_s) if norm.pre else (None, zeros)
        names = block.BlockNorm.PARAMETERS
        # post gain and bias without a norm behind the block, and pre ones without a norm, have no effect
        has = {"post_gain": norm.post, "post_bias": norm.post, "gate": 1, "pre_gain": norm.pre, "pre_bias": norm.pre}
        grads = {k: torch.empty(norm.tensors[k].shape, device=u.device) for i, k in enumerate(names)
                 if norm.tensors[k] is not None and has[k] and ctx.needs_input_grad[2 + i]}
        gu = torch.empty_like(u)
        gr = torch.empty(ctx.r_shape, dtype=u.dtype, device=u.device) if ctx.needs_input_grad[1] else None
        block.nfad_block_norm_backward(norm, grad_h.contiguous() if norm.pre else None, None if grad_s is None else grad_s.contiguous(), u, s, stats, gu, gr, grads,
                                       block.nfad_block_norm_backward_scratch(norm, u))
        return (gu, gr, *(grads[k].to(u.dtype) if k in grads else None for k in names), None, None, None, None)


def block_norm(u, r=None, post="none", pre="rms", post_gain=None, post_bias=None, gate=None, pre_gain=None, pre_bias=None,
               residual_scale: float = 1.0, eps: float = 1e-5):
    """s = residual_scale r + gate N_post(u) and h = N_pre(s), for tensors [..., cols]; see ``block.BlockNorm``.
    Returns (s, h); h is empty when pre is "none"."""
    return BlockNormFunction.apply(u, r, post_gain, post_bias, gate, pre_gain, pre_bias, post, pre, residual_scale, eps)


def _expert_grad_bias(grad, dfdx, offsets, want_bias):
    """grad dfdx (grad itself without dfdx) and, when wanted, its sums over each expert's rows."""
    gz = torch.empty_like(grad) if dfdx is not None else None
    gb = torch.empty(offsets.numel() - 1, grad.shape[1], device=grad.device) if want_bias else None
    if gz is not None or gb is not None:
        block.nfad_expert_act_backward(grad, dfdx, offsets, gz, gb, block.nfad_expert_act_backward_scratch(grad) if want_bias else None)
    return grad if gz is None else gz, gb


class ExpertLinear(torch.autograd.Function):
    """y = f(x w_e^T + b_e) for rows grouped by expert; saved: x, w and f' (no z)."""

    @staticmethod
    def forward(ctx, x, w, bias, offsets, kind):
        xc, wc, bc = x.contiguous(), w.contiguous(), None if bias is None else bias.contiguous()
        y = torch.empty(xc.shape[0], wc.shape[1], dtype=xc.dtype, device=xc.device)
        d = torch.empty_like(y) if kind is not None else None
        block.nfad_expert_linear(kind, xc, wc, bc, offsets, y, d)
        ctx.save_for_backward(xc, wc, offsets, *([] if d is None else [d]))
        ctx.bias_dtype = None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        x, w, offsets, *d = ctx.saved_tensors
        gz, gb = _expert_grad_bias(grad_out.contiguous(), d[0] if d else None, offsets, ctx.needs_input_grad[2])
        gx = gw = None
        if ctx.needs_input_grad[0]:
            gx = torch.empty_like(x)
            block.nfad_expert_linear_backward_input(gz, w, offsets, None, gx)
        if ctx.needs_input_grad[1]:
            gw = torch.empty_like(w)
            block.nfad_expert_linear_backward_weight(gz, x, offsets, gw)
        return gx, gw, None if gb is None else gb.to(ctx.bias_dtype), None, None


def expert_linear(x, w, bias, offsets, kind=None):
    """x [rows, in] sorted by expert, w [experts, out, in], bias [experts, out] or None, offsets int32 [experts + 1]."""
    return ExpertLinear.apply(x, w, bias, offsets, kind)


class ExpertFeedForward(torch.autograd.Function):
    """w2 f(w1 x + b1) + b2 for rows grouped by expert.  Saved: x, y1 = f(z1), f'(z1) and the weights; on the way back the second
    layer's input gradient leaves its product already multiplied by f'(z1) (Eq. 4 in the epilogue)."""

    @staticmethod
    def forward(ctx, x, w1, b1, w2, b2, offsets, kind):
        xc, w1c, w2c = x.contiguous(), w1.contiguous(), w2.contiguous()
        y1 = torch.empty(xc.shape[0], w1c.shape[1], dtype=xc.dtype, device=xc.device)
        d1 = torch.empty_like(y1)
        block.nfad_expert_linear(kind, xc, w1c, None if b1 is None else b1.contiguous(), offsets, y1, d1)
        y2 = torch.empty(xc.shape[0], w2c.shape[1], dtype=xc.dtype, device=xc.device)
        block.nfad_expert_linear(None, y1, w2c, None if b2 is None else b2.contiguous(), offsets, y2)
        ctx.save_for_backward(xc, y1, d1, w1c, w2c, offsets)
        ctx.bias_dtypes = [None if b is None else b.dtype for b in (b1, b2)]
        return y2

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        x, y1, d1, w1, w2, offsets = ctx.saved_tensors
        need = ctx.needs_input_grad
        g2, gb2 = _expert_grad_bias(grad_out.contiguous(), None, offsets, need[4])
        gw1 = gw2 = gx = None
        if need[3]:
            gw2 = torch.empty_like(w2)
            block.nfad_expert_linear_backward_weight(g2, y1, offsets, gw2)
        g1 = torch.empty_like(d1)
        block.nfad_expert_linear_backward_input(g2, w2, offsets, d1, g1)
        _, gb1 = _expert_grad_bias(g1, None, offsets, need[2])
        if need[1]:
            gw1 = torch.empty_like(w1)
            block.nfad_expert_linear_backward_weight(g1, x, offsets, gw1)
        if need[0]:
            gx = torch.empty_like(x)
            block.nfad_expert_linear_backward_input(g1, w1, offsets, None, gx)
        gb1, gb2 = (None if g is None else g.to(t) for g, t in zip((gb1, gb2), ctx.bias_dtypes))
        return gx, gw1, gb1, gw2, gb2, None, None


def expert_feed_forward(x, w1, b1, w2, b2, offsets, kind="gelu_erf"):
    """Two layers with the activation `kind` between them: w1 [experts, hidden, in], w2 [experts, out, hidden]."""
    return ExpertFeedForward.apply(x, w1, b1, w2, b2, offsets, kind)


def _differentiated(*tensors):
    """Whether a gradient can be asked for: else nothing is kept, and the derivatives are neither formed nor stored."""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _contiguous(t):
    return None if t is None else t.contiguous()


def _gated_layer(x, w, bias, offsets, kind, train):
    """f(a) u and, in a pass that will be differentiated, its two derivatives; contiguous tensors."""
    y = torch.empty(x.shape[0], w.shape[2], dtype=x.dtype, device=x.device)
    both = torch.empty(x.shape[0], 2, w.shape[2], dtype=x.dtype, device=x.device) if train else None
    block.nfad_expert_gated_linear(kind, x, w, bias, offsets, y, both)
    return y, both


def _second_layer(y1, w, bias, offsets):
    y = torch.empty(y1.shape[0], w.shape[1], dtype=y1.dtype, device=y1.device)
    block.nfad_expert_linear(None, y1, w, bias, offsets, y)
    return y


class ExpertGatedLinear(torch.autograd.Function):
    """y = f(a) u, a and u the products with the two weights, for rows grouped by expert; saved: x, w and y's two derivatives (no a, no u)."""

    @staticmethod
    def forward(ctx, x, w, bias, offsets, kind):
        xc, wc = x.contiguous(), w.contiguous()
        y, both = _gated_layer(xc, wc, _contiguous(bias), offsets, kind, True)
        ctx.save_for_backward(xc, wc, offsets, both)
        ctx.bias_dtype = None if bias is None else bias.dtype
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        x, w, offsets, both = ctx.saved_tensors
        gz, gb = torch.empty_like(both), None
        if ctx.needs_input_grad[2]:
            gb = torch.empty(*w.shape[:3], device=x.device)
        scratch = block.nfad_expert_act_backward_scratch(gz.flatten(1)) if gb is not None else None
        block.nfad_expert_gated_backward(grad_out.contiguous(), both, offsets, gz, gb, scratch)
        gx, gw = _gated_products(gz, x, w, offsets, ctx.needs_input_grad[:2])
        return gx, gw, None if gb is None else gb.to(ctx.bias_dtype), None, None


def _gated_products(gz, x, w, offsets, need):
    """The gradients of a gated layer's input and weights: those of a linear layer with twice the outputs."""
    gx = gw = None
    if need[0]:
        gx = torch.empty_like(x)
        block.nfad_expert_linear_backward_input(gz.flatten(1), w.flatten(1, 2), offsets, None, gx)
    if need[1]:
        gw = torch.empty_like(w)
        block.nfad_expert_linear_backward_weight(gz.flatten(1), x, offsets, gw.view(w.shape[0], -1, w.shape[3]))
    return gx, gw


def expert_gated_linear(x, w, bias, offsets, kind="swish"):
    """x [rows, in] sorted by expert, w [experts, 2, out, in] (the gate's first), bias [experts, 2, out] or None, offsets int32 [experts + 1]."""
    if not _differentiated(x, w, bias):
        return _gated_layer(x.contiguous(), w.contiguous(), _contiguous(bias), offsets, kind, False)[0]
    return ExpertGatedLinear.apply(x, w, bias, offsets, kind)


class ExpertGatedFeedForward(torch.autograd.Function):
    """w2 (f(a) u) + b2, a and u the products of x with w1's two weights.  Saved: x, y1 = f(a) u, its two derivatives and the weights; on the way
    back the second layer's input gradient leaves its product already multiplied by both, rounded once: b1's gradient sums those rounded values
    (expert_gated_linear's sums unrounded products of a gradient that was rounded before: other last bits)."""

    @staticmethod
    def forward(ctx, x, w1, b1, w2, b2, offsets, kind):
        xc, w1c, w2c = x.contiguous(), w1.contiguous(), w2.contiguous()
        y1, both = _gated_layer(xc, w1c, _contiguous(b1), offsets, kind, True)
        y2 = _second_layer(y1, w2c, _contiguous(b2), offsets)
        ctx.save_for_backward(xc, y1, both, w1c, w2c, offsets)
        ctx.bias_dtypes = [None if b is None else b.dtype for b in (b1, b2)]
        return y2

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        x, y1, both, w1, w2, offsets = ctx.saved_tensors
        need = ctx.needs_input_grad
        g2, gb2 = _expert_grad_bias(grad_out.contiguous(), None, offsets, need[4])
        gw2 = None
        if need[3]:
            gw2 = torch.empty_like(w2)
            block.nfad_expert_linear_backward_weight(g2, y1, offsets, gw2)
        gz = gb1 = gx = gw1 = None
        if any(need[:3]):
            gz = torch.empty_like(both)
            block.nfad_expert_linear_backward_gated(g2, w2, offsets, both, gz)
            _, gb1 = _expert_grad_bias(gz.flatten(1), None, offsets, need[2])
            gx, gw1 = _gated_products(gz, x, w1, offsets, need[:2])
        gb1 = None if gb1 is None else gb1.view(w1.shape[:3]).to(ctx.bias_dtypes[0])
        return gx, gw1, gb1, gw2, None if gb2 is None else gb2.to(ctx.bias_dtypes[1]), None, None


def expert_gated_feed_forward(x, w1, b1, w2, b2, offsets, kind="swish"):
    """A gated layer and a linear one: w1 [experts, 2, hidden, in] (the gate's first), w2 [experts, out, hidden]."""
    if not _differentiated(x, w1, b1, w2, b2):
        y1, _ = _gated_layer(x.contiguous(), w1.contiguous(), _contiguous(b1), offsets, kind, False)
        return _second_layer(y1, w2.contiguous(), _contiguous(b2), offsets)
    return ExpertGatedFeedForward.apply(x, w1, b1, w2, b2, offsets, kind)


class Dropout(torch.autograd.Function):
    """residual + m x; nothing is saved but what names the mask: the backward pass draws it again."""

    @staticmethod
    def forward(ctx, x, residual, drop):
        xc = x.contiguous()
        y = torch.empty_like(xc)
        block.nfad_dropout(drop, xc, None if residual is None else residual.contiguous(), y)
        ctx.numbers = drop.p, drop.seed, drop.offset
        # with autograd, which refuses a backward pass after the step has been counted up in place
        ctx.save_for_backward(*([] if drop.step is None else [drop.step]))
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        gx = None
        if ctx.needs_input_grad[0]:
            g = grad_out.contiguous()
            gx = torch.empty_like(g)
            block.nfad_dropout(block.Dropout(*ctx.numbers, *ctx.saved_tensors), g, None, gx)
        return gx, grad_out if ctx.needs_input_grad[1] else None, None


def dropout(x, drop, residual=None):
    """m x, or residual + m x, with the mask of a ``block.Dropout``."""
    if residual is not None and residual.shape != x.shape:
        raise ValueError("residual must have x's shape")
    return Dropout.apply(x, residual, drop)


class NestedBiasActivationDropout(torch.autograd.Function):
    """m f(x + bias) for x [..., cols]; m f'(x + bias) is the only saved tensor and carries the mask: the backward pass is that of the activation
    without dropout."""

    @staticmethod
    def forward(ctx, x, bias, kind, drop):
        xc = x.contiguous()
        y, d = torch.empty_like(xc), torch.empty_like(xc)
        block.nfad_bias_act_dropout_forward(kind, drop, xc, None if bias is None else bias.contiguous(), y, d)
        ctx.save_for_backward(d)
        ctx.kind, ctx.bias_dtype, ctx.cols = kind, None if bias is None else bias.dtype, xc.shape[-1] if xc.dim() else 1
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_out):
        (d,) = ctx.saved_tensors
        g = grad_out.contiguous()
        gin = torch.empty_like(g)
        if not ctx.needs_input_grad[1]:
            nfad.nfad_act_backward(ctx.kind, g.view(-1), d.view(-1), gin.view(-1))
            return gin, None, None, None
        gb = torch.empty(ctx.cols, dtype=torch.float32, device=g.device)
        nb = nfad.nfad_bias_act_backward_scratch_bytes(g.dtype, g.numel() // max(1, ctx.cols), ctx.cols, g.device)
        scratch = torch.empty(nb, dtype=torch.uint8, device=g.device) if nb else None
        nfad.nfad_bias_act_backward(ctx.kind, g.view(-1), d.view(-1), gin.view(-1), gb, scratch)
        return gin, gb.to(ctx.bias_dtype), None, None


def bias_act_dropout(x, bias, kind, drop):
    """Dropout of f(x + bias) (bias [cols] or None), with the mask of a ``block.Dropout``."""
    return NestedBiasActivationDropout.apply(x, bias, kind, drop)


def bias_gelu(x, bias, approximate: str = "none"):
    return NestedBiasActivation.apply(x, bias, "gelu_tanh" if approximate == "tanh" else "gelu_erf")


def gelu(x, approximate: str = "none"):
    return NestedActivation.apply(x, "gelu_tanh" if approximate == "tanh" else "gelu_erf")


def silu(x):
    return NestedActivation.apply(x, "swish")


def mish(x):
    return NestedActivation.apply(x, "mish")
