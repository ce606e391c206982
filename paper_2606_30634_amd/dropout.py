"""Dropout with the residual added, for torch tensors: a thin layer over the C ABI that checks arguments and passes
torch's current stream.

    h = dropout_add(branch, x, p, seed, offset)          # the mask is a function of (seed, offset, place): not stored
    dbranch = dropout_backward(dh, p, seed, offset)      # the gradient in x is dh itself

A caller draws a new offset for every call whose mask should differ.  Nothing here records for autograd."""
from __future__ import annotations

import torch

from . import binding as B
from .losses import _launch, _rows


def _run(x, residual, p, seed, offset, out):
    px, n, c, ldx, bf = _rows("x", x)
    dev = x.device
    pr, ldr = None, 0
    if residual is not None:
        pr, rn, rc, ldr, rbf = _rows("residual", residual, dev)
        if (rn, rc, rbf) != (n, c, bf):
            raise ValueError(f"x {x.dtype} {tuple(x.shape)} and residual {residual.dtype} {tuple(residual.shape)} do not match")
    if out is None:
        out = torch.empty(n, c, dtype=x.dtype, device=dev)
    po, on, oc, ldo, obf = _rows("out", out, dev)
    if (on, oc, obf) != (n, c, bf):
        raise ValueError(f"out: expected {x.dtype} of shape {(n, c)}, got {out.dtype} {(on, oc)}")
    for name, v in (("seed", seed), ("offset", offset)):
        if not isinstance(v, int) or not 0 <= v < 1 << 64:
            raise ValueError(f"{name}: expected an integer in [0, 2^64), got {v!r}")
    _launch(dev, B.dropout_add, n, c, px, ldx, pr, ldr, po, ldo, bf, p, seed, offset)
    return out


def dropout_add(x, residual, p: float, seed: int, offset: int = 0, *, out=None) -> torch.Tensor:
    """residual + x with elements of x dropped with probability p (in steps of 2^-16, at most 1 - 2^-16) and the rest
    scaled to keep its mean.  x, residual, out: [rows, cols] fp32 or bf16, rows contiguous; out may be x or residual."""
    if residual is None:
        raise ValueError("residual: expected a tensor, got None")
    return _run(x, residual, p, seed, offset, out)


def dropout_backward(dy, p: float, seed: int, offset: int = 0, *, out=None) -> torch.Tensor:
    """The gradient in x of dropout_add(x, ., p, seed, offset): the same mask and scale on dy.  (Also dropout itself,
    where there is no residual.)"""
    return _run(dy, None, p, seed, offset, out)
