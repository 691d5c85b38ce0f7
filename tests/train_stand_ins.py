"""Plain CPU stand-ins for the kernels that ``train_ops`` calls, so that its autograd side is tested
without a GPU. They refuse what the library refuses of a matrix, and count their calls."""
import contextlib

import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import train_ops as T
from tests import train_ref as ref


def _library_takes(*mats):
    for m in mats:
        rows, cols = m.shape
        if m.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("element type")
        if (cols > 1 and m.stride(1) != 1 and rows > 0) or (rows > 1 and m.stride(0) < cols):
            raise B.SignSGDError(B.SS_ERR_INVALID_ARG, "stand-in")


def _pack(x, ckpt):
    if x.numel() == 0:
        return
    codes, exps, _, _ = ref.act8(x)
    ckpt.copy_(torch.cat([codes.reshape(-1), exps.reshape(-1)]))


def decoded(ckpt, rows, cols):
    if rows * cols == 0:
        return torch.zeros(rows, cols, dtype=torch.float64)
    groups = -(-cols // ref.GROUP)
    codes, exps = ckpt[:rows * groups * ref.GROUP].long(), ckpt[rows * groups * ref.GROUP:].long()
    q = (codes & 127) * (1 - 2 * (codes >> 7))
    return (q.view(rows, groups, ref.GROUP) * ref.two_to(exps.view(rows, groups, 1) - 127)).view(rows, -1)[:, :cols]


def install(monkeypatch):
    """Replaces the kernels in ``binding``; returns the calls made, by name."""
    calls = []

    def ss_act8_pack(x, ckpt, stream=None):
        calls.append("pack")
        _library_takes(x)
        _pack(x, ckpt)

    def ss_weight_grad8(dy, ckpt_x, dw, accumulate=False, workspace=None, stream=None):
        calls.append("weight_grad")
        _library_takes(dy, dw)
        out = (dy.double().t() @ decoded(ckpt_x, dy.shape[0], dw.shape[1])).float()
        dw.detach().copy_(dw.detach() + out if accumulate else out)

    def ss_act8_forward(x, up, act, y, ckpt_x=None, ckpt_up=None, ckpt_y=None, stream=None):
        calls.append("forward")
        _library_takes(*[m for m in (x, up, y) if m is not None])
        f = ref.act("gelu" if act == B.SS_ACT_GELU else "silu", x.double())[0]
        y.copy_(f if up is None else f * up.double())
        for m, c in ((x, ckpt_x), (up, ckpt_up), (y, ckpt_y)):
            if c is not None:
                calls.append("kept")
                _pack(m, c)

    def ss_act8_backward(dy, ckpt_x, ckpt_up, act, dx, dup=None, stream=None):
        calls.append("backward")
        _library_takes(*[m for m in (dy, dx, dup) if m is not None])
        f, slope = ref.act("gelu" if act == B.SS_ACT_GELU else "silu", decoded(ckpt_x, *dy.shape))
        d = dy.double()
        if ckpt_up is None:
            dx.copy_(d * slope)
        else:
            dx.copy_(d * decoded(ckpt_up, *dy.shape) * slope)
            dup.copy_(d * f)

    def ss_policy_loss(logits, targets, old_logp, ref_logp, advantages, weights, totals, logp, dlogits=None,
                       inv_temperature=1.0, clip_low=0.2, clip_high=0.2, kl_coef=0.0, grad_scale=None, workspace=None, stream=None):
        calls.append("policy")
        _library_takes(logits)
        t, lp, d = ref.policy(logits.detach(), targets, old_logp, ref_logp, advantages, weights, inv_temperature, clip_low, clip_high, kl_coef)
        totals.copy_(t)
        logp.copy_(lp)
        if dlogits is not None:
            dlogits.copy_(d * (1.0 if grad_scale is None else grad_scale.double()))

    def ss_preference_loss(logits, targets, weights, seq_begin, ref_seq_logp, loss, margins, seq_logp, logp, dlogits=None,
                           inv_temperature=1.0, kind=0, beta=0.1, label_smoothing=0.0, scale=1.0, grad_scale=None,
                           workspace=None, stream=None):
        calls.append("preference")
        _library_takes(logits)
        out = ref.preference(logits.detach(), targets, weights, seq_begin, ref_seq_logp, inv_temperature, kind, beta, label_smoothing, scale)
        for to, of in zip((loss, margins, seq_logp, logp), out):
            to.copy_(of.reshape(to.shape))
        if dlogits is not None:
            dlogits.copy_(out[4] * (1.0 if grad_scale is None else grad_scale.double()))

    for f in (ss_act8_pack, ss_weight_grad8, ss_act8_forward, ss_act8_backward, ss_policy_loss, ss_preference_loss):
        monkeypatch.setattr(B, f.__name__, f)
    monkeypatch.setattr(T, "_in_order", lambda node, g: contextlib.nullcontext())  # streams
    return calls
