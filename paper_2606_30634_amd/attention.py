"""Attention over a range of keys per query, and the key ranges of packed documents, for torch tensors: a thin layer
over the C ABI that checks arguments, allocates what the caller does not hand over and passes torch's current
stream.  No arithmetic happens here; every step runs in the library's kernels.

    start, end = key_ranges(documents, prefix=flags)          # once per batch, for every block
    fwd = attention(q, k, v, key_start=start, key_end=end, softcap=50.0, keep_f32=True)
    dq, dk, dv = attention_backward(q, k, v, fwd, dout, key_start=start, key_end=end, softcap=50.0)

    step = attention(q1, cache_k, cache_v, q_start=lengths)   # new tokens behind answers of different lengths

Outputs go into the tensors of `out` where given.  `workspace`, a uint8 tensor of at least the matching
workspace_bytes of the binding, is allocated per call where not given.  Nothing here records for autograd."""
from __future__ import annotations

import math
from typing import NamedTuple, Optional

import torch

from . import binding as B
from .losses import _F32, _I32, _U8, _launch, _out, _ptr, _require, _workspace

_DTYPES = (torch.float32, torch.bfloat16)


class Attention(NamedTuple):
    o: Optional[torch.Tensor] = None      # [B, Sq, H, hd]
    lse: Optional[torch.Tensor] = None    # [B, H, Sq] fp32; -inf where a query sees no key
    o_f32: Optional[torch.Tensor] = None  # o before its rounding to bf16, where it is kept


def key_ranges(documents, *, prefix=None, out=None):
    """(key_start, key_end) [B, S] int32 of packed documents: query i sees the keys [key_start, key_end) of its
    row.  documents [B, S] int32: a document is a run of equal ids >= 0, ids below 0 are padding, which
    sees nothing.  A token sees its document up to itself; the flagged tokens (prefix [B, S] bool or
    uint8) that a document starts with see all of each other."""
    if not isinstance(documents, torch.Tensor) or documents.dim() != 2 or not documents.is_cuda:
        raise ValueError("documents: expected an int32 [B, S] tensor on a GPU")
    dev, shape = documents.device, documents.shape
    ids = _require("documents", documents, dev, _I32, shape)
    flags = None
    if prefix is not None:
        if getattr(prefix, "dtype", None) is torch.bool:
            prefix = prefix.view(_U8)
        flags = _require("prefix", prefix, dev, _U8, shape)
    start, end = out if out is not None else (None, None)
    start, end = _out("key_start", start, dev, _I32, shape), _out("key_end", end, dev, _I32, shape)
    _launch(dev, B.attention_key_ranges, shape[0], shape[1], ids, flags, start.data_ptr(), end.data_ptr())
    return start, end


def _heads(name, t, dev=None, dtype=None, shape=None):
    """(pointer, strides) of rows [B, S, H, hd] whose heads are contiguous"""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a tensor, got {type(t).__name__}")
    if (t.dim() != 4 or t.dtype not in _DTYPES or not t.is_cuda or (dev is not None and t.device != dev)
            or (dtype is not None and t.dtype != dtype) or (shape is not None and t.shape != shape)):
        raise ValueError(f"{name}: expected {dtype or 'a float32 or bfloat16 tensor'} {tuple(shape or ('B', 'S', 'H', 'hd'))} "
                         f"on {dev or 'a GPU'}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    sb, ss, sh, sd = t.stride()
    nb, ns, nh, nd = t.shape
    if sd != 1 and nd > 1:
        raise ValueError(f"{name}: the elements of a head must be contiguous, got strides {t.stride()}")
    # the stride of a dimension of one is never used, and torch leaves it anything
    return t.data_ptr(), B._STRIDES(sb if nb > 1 else 0, ss if ns > 1 else 0, sh if nh > 1 else 0)


def _params(q, k, v, key_start, key_end, q_start, scale, softcap, slopes):
    pq, sq = _heads("q", q)
    dev, dtype = q.device, q.dtype
    b, nq, h, hd = q.shape
    pk, sk = _heads("k", k, dev, dtype)
    if k.shape[0] != b or k.shape[3] != hd:
        raise ValueError(f"q {tuple(q.shape)} and k {tuple(k.shape)} do not match")
    pv, sv = _heads("v", v, dev, dtype, k.shape)
    rows = torch.Size((b, nq))
    start = None if key_start is None else _require("key_start", key_start, dev, _I32, rows)
    end = None if key_end is None else _require("key_end", key_end, dev, _I32, rows)
    first = None if q_start is None else _require("q_start", q_start, dev, _I32, torch.Size((b,)))
    slope = None if slopes is None else _require("slopes", slopes, dev, _F32, torch.Size((h,)))
    params = B.AttentionParams(b, nq, k.shape[1], h, k.shape[2], hd, dtype is torch.bfloat16, sq, sk, sv, start, end,
                               first, slope, 1.0 / math.sqrt(hd) if scale is None else scale, softcap)
    return params, pq, pk, pv, dev


def attention(q, k, v, *, key_start=None, key_end=None, q_start=None, scale: Optional[float] = None,
              softcap: float = 0.0, slopes=None, keep_f32: bool = False, out: Optional[Attention] = None,
              workspace=None) -> Attention:
    """Softmax attention of q [B, Sq, H, hd] over k, v [B, Sk, KV, hd] (fp32 or bf16; any strides whose heads are
    contiguous and 16-byte aligned; KV divides H; hd 32, 64 or 128).  Query i has position q_start[b] + i ([B]
    int32; Sk - Sq without it) and sees the keys [key_start, key_end) ([B, Sq] int32), or those at or before its
    position.  softcap > 0 caps the scores scale q.k at +-softcap by a tanh; slopes [H] fp32 lowers them by
    slope |position - key|.  keep_f32: also o in fp32, for the backward of a bf16 attention."""
    params, pq, pk, pv, dev = _params(q, k, v, key_start, key_end, q_start, scale, softcap, slopes)
    b, nq, h, _ = q.shape
    out = out or Attention()
    bf = q.dtype is torch.bfloat16
    if out.o_f32 is not None and not (keep_f32 and bf):
        raise ValueError("out.o_f32 needs keep_f32, and bfloat16 inputs")
    out = Attention(_out("o", out.o, dev, q.dtype, q.shape), _out("lse", out.lse, dev, _F32, (b, h, nq)),
                    _out("o_f32", out.o_f32, dev, _F32, q.shape) if keep_f32 and bf else None)
    ws, nb = _workspace(workspace, B.attention_workspace_bytes(params), dev)
    _launch(dev, B.attention_forward, params, pq, pk, pv, out.o.data_ptr(), _ptr(out.o_f32), out.lse.data_ptr(),
            _ptr(ws), nb)
    return out


def attention_backward(q, k, v, forward: Attention, dout, *, key_start=None, key_end=None, q_start=None,
                       scale: Optional[float] = None, softcap: float = 0.0, slopes=None, out=None, workspace=None):
    """(dq, dk, dv) of attention(), from its inputs, its outputs (o_f32 where it was kept, else o; lse) and the gradient
    dout [B, Sq, H, hd] in o.  out: the three, of the inputs' shapes and type, any strides as in attention()."""
    params, pq, pk, pv, dev = _params(q, k, v, key_start, key_end, q_start, scale, softcap, slopes)
    b, nq, h, _ = q.shape
    wide = forward.o_f32 is not None
    po, so = _heads("forward.o_f32", forward.o_f32, dev, _F32, q.shape) if wide else _heads("forward.o", forward.o, dev, q.dtype, q.shape)
    lse = _require("forward.lse", forward.lse, dev, _F32, torch.Size((b, h, nq)))
    pd, sd = _heads("dout", dout, dev, q.dtype, q.shape)
    if out is None:
        out = tuple(torch.empty(t.shape, dtype=t.dtype, device=dev) for t in (q, k, v))
    dq, dk, dv = out
    (gq, tq), (gk, tk), (gv, tv) = (_heads("out", g, dev, q.dtype, t.shape) for g, t in ((dq, q), (dk, k), (dv, v)))
    grads = B.AttentionGrads(so, sd, tq, tk, tv, gq, gk, gv, wide)
    ws, nb = _workspace(workspace, B.attention_backward_workspace_bytes(params), dev)
    _launch(dev, B.attention_backward, params, pq, pk, pv, po, lse, pd, grads, _ptr(ws), nb)
    return dq, dk, dv
