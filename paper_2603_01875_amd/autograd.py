"""torch.autograd front end of the library: the losses as differentiable scalars.

The forward call runs the whole fused path (loss AND both gradients come out of one
call of the library); backward only scales the stored gradients by the incoming scalar (the one
PyTorch op here: the chain rule through whatever the caller does with the loss).  No step of the
method runs in PyTorch: this module is argument marshalling, like kdloss.py.
"""
from __future__ import annotations

import torch

from . import kdloss as K


def _scaled(x, g, dtype=None):
    """x times the scalar tensor g, in fp32 with one rounding to `dtype` (x's type).  (g rounded to bf16 first would shift all of a gradient the
    same way, and torch rounds a scalar tensor on the device to the other operand's type.  One pass, of [151936, 1024] in bf16
    141 us; 120 with g rounded.)"""
    if x is None:
        return None
    if torch.is_grad_enabled() and g.requires_grad:        # (a graph of the backward pass: the factor's part in it)
        return (x.float() * g).to(dtype or x.dtype)
    return torch.mul(x, g.reshape(1), out=torch.empty_like(x, dtype=dtype))


class _KDLossFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h_s, W_s, h_t, W_t, mask, tau, kind, beta, w_layout, flags, teacher_scale, workspace,
                loss_scale):
        out = K.kd_loss_fwd_bwd(h_t, W_t, h_s, W_s, mask, tau=tau, kind=kind, beta=beta, w_layout=w_layout,
                                workspace=workspace, want_per_token=False, flags=flags,
                                teacher_scale=teacher_scale, loss_scale=loss_scale)
        ctx.save_for_backward(out["grad_h_s"], out["grad_W_s"])
        return out["loss"].reshape(())

    @staticmethod
    def backward(ctx, g):
        return tuple(_scaled(x, g) for x in ctx.saved_tensors) + (None,) * 11


def kd_loss(h_s, W_s, h_t, W_t, mask=None, tau=1.0, kind=K.FKL, beta=0.5, w_layout=K.W_VH, flags=0,
            teacher_scale=0.0, workspace=None, loss_scale=1.0):
    """Masked-mean divergence between softmax(h_t W_t / tau) and softmax(h_s W_s / tau) as a scalar
    tensor; gradients flow to h_s and W_s (the teacher side is frozen).  Arguments as in
    kdloss.kd_loss_fwd_bwd.  A factor that is known before the call (1 / micro-batches, a loss weight)
    belongs in `loss_scale`: the library folds it into the loss and both gradients at no cost, whereas
    whatever multiplies the returned scalar afterwards costs backward() one more pass over the
    gradients (they are formed in forward, before that factor exists)."""
    return _KDLossFn.apply(h_s, W_s, h_t, W_t, mask, float(tau), int(kind), float(beta), int(w_layout),
                           int(flags), float(teacher_scale), workspace, float(loss_scale))


class _HeadLossFn(torch.autograd.Function):
    """A one-head loss: `call(want_grad_h, want_grad_W)` gives the dict of a *_fwd_bwd call.  Only the gradients that are asked
    for are computed.  They may have another type than h and W: backward rounds them to theirs with its product."""

    @staticmethod
    def forward(ctx, h, W, call, names):
        out = call(ctx.needs_input_grad[0], ctx.needs_input_grad[1])
        ctx.save_for_backward(out[names[0]], out[names[1]])
        ctx.types = (h.dtype, W.dtype)
        return out["loss"].reshape(())

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, g):
        return tuple(_scaled(x, g, t) for x, t in zip(ctx.saved_tensors, ctx.types)) + (None, None)


def cross_entropy(h, W, labels, mask=None, label_smoothing=0.0, z_loss=0.0, w_layout=K.W_VH, workspace=None,
                  loss_scale=1.0, grad_dtype=None):
    """Cross entropy of `labels` (negative: ignored) under softmax(h W) as a scalar tensor, the mean over the tokens that
    count; gradients flow to h and W.  Arguments as in kdloss.kd_ce_fwd_bwd; loss_scale as in kd_loss.  Where no gradient is
    asked for, none is computed.  grad_dtype=kdloss.F32 with bf16 h and W: what the library computes and keeps for backward() is
    fp32, and the gradients are rounded to bf16 once, by backward(); by default dL/dz is rounded to bf16 as well, in half the
    time (T = 4096, H = 1024, V = 151936 4.2 ms, 9.0 in fp32).  (A workspace that is given has to be one for the same grad_dtype.)"""
    kw = dict(label_smoothing=float(label_smoothing), z_loss=float(z_loss), w_layout=int(w_layout), workspace=workspace,
              loss_scale=float(loss_scale))
    if not (torch.is_grad_enabled() and (h.requires_grad or W.requires_grad)):
        return K.kd_ce_fwd(h.detach(), W.detach(), labels, mask, **kw)["loss"].reshape(())
    return _HeadLossFn.apply(h, W, lambda gh, gW: K.kd_ce_fwd_bwd(h.detach(), W.detach(), labels, mask, grad_dtype=grad_dtype,
                                                                  want_grad_h=gh, want_grad_W=gW, **kw), ("grad_h", "grad_W"))


def topk_loss(h_s, W_s, top_logits, top_index, lse=None, mask=None, tau=1.0, tail=K.TAIL_RENORM, w_layout=K.W_VH, flags=0,
              workspace=None, loss_scale=1.0, grad_dtype=None):
    """Divergence of softmax(h_s W_s / tau) from a teacher's top logits as a scalar tensor; gradients flow to h_s and W_s.
    Arguments as in kdloss.kd_topk_fwd_bwd; loss_scale as in kd_loss, grad_dtype as in cross_entropy.  Where no gradient is asked
    for, none is computed."""
    kw = dict(lse=lse, mask=mask, tau=float(tau), tail=int(tail), w_layout=int(w_layout), flags=int(flags),
              workspace=workspace, loss_scale=float(loss_scale))
    if not (torch.is_grad_enabled() and (h_s.requires_grad or W_s.requires_grad)):
        return K.kd_topk_fwd(top_logits, top_index, h_s.detach(), W_s.detach(), **kw)["loss"].reshape(())
    return _HeadLossFn.apply(h_s, W_s, lambda gh, gW: K.kd_topk_fwd_bwd(top_logits, top_index, h_s.detach(), W_s.detach(),
                                                                        grad_dtype=grad_dtype, want_grad_h=gh, want_grad_W=gW,
                                                                        **kw), ("grad_h_s", "grad_W_s"))
