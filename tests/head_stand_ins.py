"""Plain CPU stand-ins for the kernels of the cross entropy at the head and of the orthogonal update, so that what calls them is
tested without a GPU. They refuse what the library refuses of a matrix, and count their calls."""
import contextlib

import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import train_ops as T
from tests import head_ref, ortho_ref


def _library_takes(*mats):
    for m in mats:
        rows, cols = m.shape
        if m.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("element type")
        if (cols > 1 and m.stride(1) != 1 and rows > 0) or (rows > 1 and m.stride(0) < cols):
            raise B.SignSGDError(B.SS_ERR_INVALID_ARG, "stand-in")


def ss_linear_cross_entropy(calls, x, weight, targets, weights, totals, logp, dx=None, dw=None, accumulate=False, inv_temperature=1.0,
                            z_coef=0.0, grad_scale=None, workspace=None, stream=None):
    calls.append(("head", dx is not None, dw is not None))
    _library_takes(*[m for m in (x, weight, dx, dw) if m is not None])
    assert x.dtype == weight.dtype and targets.dim() == weights.dim() == 1
    assert dw is None or dw.dtype == torch.float32 or (x.dtype == torch.bfloat16 and not accumulate)
    out = head_ref.head(x.detach(), weight.detach(), targets, weights, inv_temperature, z_coef, 1.0 if grad_scale is None else float(grad_scale))
    totals.copy_(out["totals"])
    logp.copy_(out["logp"])
    if dx is not None:
        dx.copy_(out["dx"])
    if dw is not None:
        dw.copy_(out["dw"] + dw if accumulate else out["dw"])


class Kernels:
    """The part of the binding that ``optim.OrthogonalMomentum`` calls."""
    SS_ORTHO_MAX_MATRICES = 4
    ORTHO_COEFFICIENTS = B.ORTHO_COEFFICIENTS

    def __init__(self):
        self.calls = []

    def ss_orthogonal_update(self, grads, momenta, momenta_out, params, params_out, beta, nesterov, coefficients, lr, scale, weight_decay):
        self.calls.append((len(grads), tuple(grads[0].shape)))
        assert 0 < len(grads) <= self.SS_ORTHO_MAX_MATRICES
        for mats in (grads, momenta, momenta_out, params, params_out):
            _library_takes(*mats)
            assert len({(m.shape, m.stride(0) if m.shape[0] > 1 else 0, m.dtype) for m in mats}) == 1
        for g, v, vo, p, po in zip(grads, momenta, momenta_out, params, params_out):
            nv, np_ = ortho_ref.updated(g, v, p, beta, nesterov, lr, scale, weight_decay, coefficients)
            vo.copy_(nv)
            po.copy_(np_)


def install(monkeypatch):
    calls = []
    monkeypatch.setattr(B, "ss_linear_cross_entropy", lambda *a, **k: ss_linear_cross_entropy(calls, *a, **k))
    monkeypatch.setattr(T, "_in_order", lambda node, g: contextlib.nullcontext())  # streams
    return calls
