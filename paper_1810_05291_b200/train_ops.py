"""The training operators as autograd functions: linear layers and activations that keep their
inputs in 8 bits for the backward pass, losses over logits, and the loss at the head that takes the
product with the head's weight in.

They make the gradients that ``optim.SignumVote`` compresses: a linear layer's weight gradient goes
to the parameter's ``grad``, which under ``SignumVote`` is a view of the flat buffer that the vote
reads, through autograd or, where the layer is asked to, straight. The layers' matrix products with
the weights are PyTorch's; everything else of the two passes is in the kernels of ``binding``
(``include/signsgd_train.h`` has the formulas). The kernels have no second derivatives: a backward
pass through the backward pass raises.
"""

from __future__ import annotations

import contextlib
import functools
import math
from typing import Optional, Tuple

import torch

from . import binding as B

ACTIVATIONS = {"gelu": B.SS_ACT_GELU, "silu": B.SS_ACT_SILU}
PREFERENCES = {"sigmoid": B.SS_PREF_SIGMOID, "hinge": B.SS_PREF_HINGE, "squared": B.SS_PREF_SQUARED}


def _rows(x: torch.Tensor) -> torch.Tensor:
    """[..., cols] as a matrix that the library takes: unit column stride, rows that do not overlap (``x``
    itself or a view where that is possible, not for the broadcast gradient of a sum over rows, say)."""
    m = x if x.dim() == 2 else x.reshape(math.prod(x.shape[:-1]), x.shape[-1])
    fits = (m.stride(1) == 1 or m.shape[1] < 2) and (m.stride(0) >= m.shape[1] or m.shape[0] < 2)
    return m if fits else m.contiguous()


def _grad_buffer(ctx, weight: torch.Tensor) -> Optional[torch.Tensor]:
    """``weight.grad``, if the kernel may add to it in autograd's place: a matrix that it takes, of a
    weight that this backward pass accumulates into, and whose gradient nothing looks at on its way or later."""
    if ctx.create_graph or not weight.is_leaf or weight._backward_hooks or weight._post_accumulate_grad_hooks:
        return None
    g = weight.grad
    if g is None or g.dtype != torch.float32 or g.dim() != 2 or g.requires_grad or _rows(g) is not g:
        return None
    try:  # whether autograd will run the node that accumulates: not for autograd.grad, nor for other inputs alone
        return g if torch._C._will_engine_execute_node(ctx.next_functions[1][0]) else None
    except RuntimeError:  # autograd.grad with respect to the weight: the gradient is to be returned
        return None


@contextlib.contextmanager
def _in_order(node, g: torch.Tensor):
    """Around a kernel that adds to ``g`` in the place of ``node``, autograd's node that accumulates there. Autograd
    orders streams for the gradients that it hands on only. So the kernel comes after others that did the same on
    another stream in this pass, and the node's stream, which the caller's waits for, comes after all of them."""
    stream, pending = torch.cuda.current_stream(g.device), node.metadata
    before = pending.get(_in_order)
    if before is not None:
        stream.wait_event(before)
    yield
    g.record_stream(stream)
    pending[_in_order] = stream.record_event()
    if before is None:
        def wait(_):
            torch.cuda.current_stream(g.device).wait_event(pending.pop(_in_order))
            handle.remove()
        handle = node.register_prehook(wait)


class _NoSecond(torch.autograd.Function):
    @staticmethod
    def forward(ctx, g):
        return g.view_as(g)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("the training operators have no second derivatives")


def _first_derivative(backward):
    """A backward pass whose results are not constants, though they carry no graph: under ``create_graph`` a
    backward pass that reaches them raises. (``once_differentiable`` lets them pass for constants where the
    gradient that arrives is one, as that of a sum is.) It is called with a gradient of its first result; the
    others have none, and no zeros are made for them (the forward pass says so)."""
    @functools.wraps(backward)
    def run(ctx, *grads):
        if grads[0] is None:
            return (None,) * len(ctx.needs_input_grad)
        ctx.create_graph = torch.is_grad_enabled()
        with torch.no_grad():
            out = backward(ctx, *grads)
        if not ctx.create_graph:
            return out
        return tuple(None if g is None else _NoSecond.apply(g.requires_grad_()) for g in out)
    return run


def _brought(kept: torch.Tensor, m: torch.Tensor) -> torch.Tensor:
    """A caller's checkpoint of ``m``, checked while the caller is there to see it."""
    if kept.dtype != torch.uint8:
        raise TypeError("kept must be uint8, got %s" % kept.dtype)
    size = B.ss_act8_bytes(*m.shape)
    if kept.shape != (size,) or not kept.is_contiguous() or kept.device != m.device or kept.data_ptr() % 16:
        raise ValueError("kept must be a contiguous, 16-byte aligned tensor of %d bytes on %s, the checkpoint of [%d, %d]"
                         % (size, m.device, *m.shape))
    return kept


class _Linear8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, kept, into_grad, wanted):
        ctx.set_materialize_grads(False)
        m = _rows(x)
        if kept is not None:
            kept = _brought(kept, m)
        elif wanted:
            kept = B.act8_checkpoint(m.shape[0], m.shape[1], m.device)
            B.ss_act8_pack(m, kept)
        w = weight.to(x.dtype)
        ctx.weight, ctx.shape, ctx.into_grad = weight, x.shape, into_grad
        # with their versions: what is written again in between is refused
        ctx.save_for_backward(w if ctx.needs_input_grad[0] else None, kept if wanted else None)
        return (m @ w.t()).view(*x.shape[:-1], weight.shape[0])

    @staticmethod
    @_first_derivative
    def backward(ctx, dy):
        weight, d = ctx.weight, _rows(dy)
        w, kept = ctx.saved_tensors
        dx = None
        if ctx.needs_input_grad[0]:
            with torch.autocast(d.device.type, enabled=False):  # in the types of the forward pass
                dx = (d @ w).view(ctx.shape)
        dw = None
        if ctx.needs_input_grad[1]:
            into = _grad_buffer(ctx, weight) if ctx.into_grad else None
            if into is not None:                  # no second buffer, no addition afterwards
                with _in_order(ctx.next_functions[1][0], into):
                    B.ss_weight_grad8(d, kept, into, accumulate=True)
            else:
                dw = torch.empty(weight.shape, dtype=torch.float32, device=weight.device)
                B.ss_weight_grad8(d, kept, dw)
        return dx, dw, None, None, None


class _Act8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, up, act, keep_output, wanted):
        ctx.set_materialize_grads(False)
        m, u = _rows(x), None if up is None else _rows(up)
        new = lambda: B.act8_checkpoint(m.shape[0], m.shape[1], m.device)  # noqa: E731
        y = torch.empty(m.shape, dtype=m.dtype, device=m.device)
        ctx.act, ctx.shape = act, x.shape
        kept, kept_up = new() if wanted else None, new() if wanted and u is not None else None
        kept_y = new() if keep_output else None
        B.ss_act8_forward(m, u, act, y, kept, kept_up, kept_y)
        ctx.save_for_backward(kept, kept_up)
        if kept_y is not None:
            ctx.mark_non_differentiable(kept_y)
        return y.view(x.shape), kept_y

    @staticmethod
    @_first_derivative
    def backward(ctx, dy, _):
        d = _rows(dy)
        dx = torch.empty(d.shape, dtype=d.dtype, device=d.device)
        kept, kept_up = ctx.saved_tensors
        dup = None if kept_up is None else torch.empty_like(dx)
        B.ss_act8_backward(d, kept, kept_up, ctx.act, dx, dup)
        return dx.view(ctx.shape), None if dup is None else dup.view(ctx.shape), None, None, None


def linear8(x: torch.Tensor, weight: torch.Tensor, kept: Optional[torch.Tensor] = None,
            into_grad: bool = False) -> torch.Tensor:
    """``x @ weight.T`` whose input is kept in 8 bits (33 bytes for 32 values) for the weight
    gradient, if one can be asked for. ``x``: [..., n_in] bfloat16 or float32; ``weight``: [n_out, n_in]
    float32, used in ``x``'s type (under autocast both are used in the region's, as in other linear
    layers). ``kept``: the checkpoint of ``x``, if it is at hand (``act8`` makes its output's); its
    contents are needed until the backward pass, which refuses one that was written again.

    The weight's gradient is handed on to autograd. With ``into_grad`` the kernel adds it to
    ``weight.grad`` itself, without a buffer in between, in a backward pass that accumulates there
    anyway; where there is no float32 ``weight.grad`` yet, or the weight has hooks, or the pass was
    asked for other gradients, it is handed on as well. (Hooks on the node that accumulates, which
    autograd does not show, are called without a gradient.)"""
    if torch.is_autocast_enabled(x.device.type) and x.dtype != torch.float64:
        x = x.to(torch.get_autocast_dtype(x.device.type))
    return _Linear8.apply(x, weight, kept, into_grad, torch.is_grad_enabled() and weight.requires_grad)


def act8(x: torch.Tensor, up: Optional[torch.Tensor] = None, act: str = "silu",
         keep_output: bool = False) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """``f(x)`` or ``f(x) * up`` whose inputs are kept in 8 bits, if a gradient can be asked for.
    Returns the result and, with ``keep_output``, its checkpoint for the ``linear8`` that follows
    (else None)."""
    wanted = torch.is_grad_enabled() and (x.requires_grad or (up is not None and up.requires_grad))
    return _Act8.apply(x, up, ACTIVATIONS[act], keep_output, wanted)


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, old_logp, ref_logp, advantages, weights, inv_temperature, clip_low, clip_high, kl_coef):
        ctx.set_materialize_grads(False)
        z = _rows(logits)
        args = (z, targets, old_logp, ref_logp, advantages, weights)
        ctx.save_for_backward(*args)
        ctx.options = dict(inv_temperature=inv_temperature, clip_low=clip_low, clip_high=clip_high, kl_coef=kl_coef)
        ctx.shape = logits.shape
        totals, logp = torch.empty(3, device=z.device), torch.empty(z.shape[0], device=z.device)
        B.ss_policy_loss(*args, totals, logp, None, **ctx.options)
        loss, rest = totals[0].clone(), totals[1:]
        ctx.mark_non_differentiable(rest, logp)
        return loss, rest, logp

    @staticmethod
    @_first_derivative
    def backward(ctx, g, *_):
        z = ctx.saved_tensors[0]
        dz, totals, logp = torch.empty_like(z), torch.empty(3, device=z.device), torch.empty(z.shape[0], device=z.device)
        B.ss_policy_loss(*ctx.saved_tensors, totals, logp, dz, grad_scale=g.reshape(1).float(), **ctx.options)
        return (dz.view(ctx.shape),) + (None,) * 9


def _preference_outputs(args):
    z, ref = args[0], args[4]
    new = lambda n: torch.empty(n, device=z.device)  # noqa: E731
    return new(1), new(ref.shape[0] // 2), new(ref.shape[0]), new(z.shape[0])


class _PreferenceLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, targets, weights, seq_begin, ref_seq_logp, options):
        ctx.set_materialize_grads(False)
        z = _rows(logits)
        args = (z, targets, weights, seq_begin, ref_seq_logp)
        ctx.save_for_backward(*args)
        ctx.options, ctx.shape = options, logits.shape
        outs = _preference_outputs(args)
        B.ss_preference_loss(*args, *outs, None, **options)
        loss = outs[0].reshape(())
        ctx.mark_non_differentiable(*outs[1:])
        return (loss,) + outs[1:]

    @staticmethod
    @_first_derivative
    def backward(ctx, g, *_):
        args = ctx.saved_tensors
        dz = torch.empty_like(args[0])
        B.ss_preference_loss(*args, *_preference_outputs(args), dz, grad_scale=g.reshape(1).float(), **ctx.options)
        return dz.view(ctx.shape), None, None, None, None, None


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, targets, weights, inv_temperature, z_coef, into_grad, want_dx, want_dw):
        ctx.set_materialize_grads(False)
        m, w = _rows(x), _rows(weight.to(x.dtype))
        totals, logp = torch.empty(2, device=m.device), torch.empty(m.shape[0], device=m.device)
        dx = torch.empty(m.shape, dtype=m.dtype, device=m.device) if want_dx else None
        dw = torch.empty(w.shape, dtype=weight.dtype if m.dtype is torch.bfloat16 else torch.float32, device=m.device) if want_dw else None
        B.ss_linear_cross_entropy(m, w, targets, weights, totals, logp, dx, dw, inv_temperature=inv_temperature, z_coef=z_coef)
        ctx.weight, ctx.shape, ctx.into_grad = weight, x.shape, into_grad
        ctx.save_for_backward(dx, dw)
        loss, square = totals[0].clone(), totals[1].clone()
        ctx.mark_non_differentiable(square, logp)
        return loss, square, logp

    @staticmethod
    @_first_derivative
    def backward(ctx, g, *_):
        (dx, dw), weight, g = ctx.saved_tensors, ctx.weight, g.float()
        if dx is not None:
            dx = _times(dx, g, dx.dtype).view(ctx.shape)
        if dw is not None:
            into = _grad_buffer(ctx, weight) if ctx.into_grad and dw.dtype is torch.float32 else None
            if into is not None:
                with _in_order(ctx.next_functions[1][0], into):
                    into.addcmul_(dw, g)
                dw = None
            else:
                dw = _times(dw, g, weight.dtype)
        return dx, dw, None, None, None, None, None, None, None


def _times(t: torch.Tensor, g: torch.Tensor, dtype) -> torch.Tensor:
    """``t * g`` in 32 bits, rounded once; some rows at a time, so that no 32-bit copy of a large gradient is made. (A
    product of a bfloat16 tensor and a scalar in device memory would round the scalar first.)"""
    if t.dtype is torch.float32 and dtype is torch.float32:
        return t * g
    out = torch.empty(t.shape, dtype=dtype, device=t.device)
    step = max(1, (1 << 26) // max(t.shape[1], 1))
    for a, b in zip(t.split(step), out.split(step)):
        b.copy_(a.float() * g)
    return out


def linear_cross_entropy(x, weight, targets, weights, inv_temperature: float = 1.0, z_coef: float = 0.0, into_grad: bool = False):
    """Softmax cross entropy of ``x @ weight.T`` at ``targets``, each position counting ``weights``, whose logits are never
    kept. ``x``: [..., width] bfloat16 or float32; ``weight``: [vocab, width] float32 or bfloat16, used in ``x``'s type
    (under autocast both in the region's); ``targets``, ``weights``: one for each position. Returns the loss, the weighted
    sum of lse^2 (``z_coef`` times it is in the loss) and the positions' log probabilities.

    Where gradients can be asked for they are formed with the loss, in one go: that takes three products with the
    head, where forming the logits again in the backward pass would take four. They are held until the backward pass, which
    multiplies them by the gradient that arrives, in 32 bits; those in bfloat16 are rounded when they are formed and again there (which
    changes nothing where that gradient is a power of two). With ``into_grad`` it adds the weight's to ``weight.grad`` itself, as in
    ``linear8``, out of the fp32 one that it holds."""
    if torch.is_autocast_enabled(x.device.type) and x.dtype != torch.float64:
        x = x.to(torch.get_autocast_dtype(x.device.type))
    on = torch.is_grad_enabled()
    return _LinearCrossEntropy.apply(x, weight, targets.reshape(-1), weights.reshape(-1), inv_temperature, z_coef, into_grad,
                                     on and x.requires_grad, on and weight.requires_grad)


def policy_loss(logits, targets, old_logp, advantages, weights, ref_logp=None, kl_coef: float = 0.0,
                clip_low: float = 0.2, clip_high: float = 0.2, inv_temperature: float = 1.0):
    """Clipped policy loss with a KL term over ``logits`` [rows, vocab]. Returns the loss, two
    figures (the weighted sum of the KL terms, the weight of the clipped positions) and the log
    probabilities. The forward pass forms no gradient; a loop of its own that wants loss and
    gradient in one pass over the logits calls ``binding.ss_policy_loss`` with ``dlogits``."""
    return _PolicyLoss.apply(logits, targets, old_logp, ref_logp, advantages, weights, inv_temperature, clip_low, clip_high, kl_coef)


def preference_loss(logits, targets, weights, seq_begin, ref_seq_logp, kind: str = "sigmoid", beta: float = 0.1,
                    label_smoothing: float = 0.0, scale: Optional[float] = None, inv_temperature: float = 1.0):
    """Preference loss over pairs of packed sequences: sequence ``s`` covers rows
    ``seq_begin[s] : seq_begin[s + 1]``, ``2 p`` is the preferred one of pair ``p``. ``scale``
    defaults to the mean over the pairs. Returns the loss, the margins, the sequences' log
    probabilities and the positions' log probabilities."""
    pairs = ref_seq_logp.shape[0] // 2
    return _PreferenceLoss.apply(logits, targets, weights, seq_begin, ref_seq_logp,
                                 dict(kind=PREFERENCES[kind], beta=beta, label_smoothing=label_smoothing,
                                      scale=1.0 / max(pairs, 1) if scale is None else scale,
                                      inv_temperature=inv_temperature))
