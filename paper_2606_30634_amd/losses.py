"""Log-probabilities and the losses on them, for torch tensors: a thin layer over the C ABI that checks
arguments, allocates what the caller does not hand over and passes torch's current stream.  No arithmetic
happens here; every step runs in the library's kernels.

    lp = token_logprob(logits, targets)                       # or head_logprob(hidden, head, targets)
    out = policy_loss(lp.logp.view(B, S), old, advantages, mask, ref_logp=ref, kl_coef=0.05)
    dlogits = token_logprob_backward(logits, targets, lp, out.dlogp.view(-1))

A function writes into the tensors of `out` where given (fields that are None are allocated where the
operator needs them) and returns its outputs.  `workspace`, a uint8 tensor of at least the matching
workspace_bytes of the binding, is allocated per call where not given.

Nothing here records for autograd: outputs are detached whatever the inputs ask for, and a gradient is one of the
functions above (head_logprob has none)."""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as B

_F32, _BF16, _I32, _U8 = torch.float32, torch.bfloat16, torch.int32, torch.uint8
_KINDS = {"sigmoid": 0, "hinge": 1, "square": 2}
_REDUCTIONS = {"token": 0, "sequence": 1}


# The current stream's handle of a device: torch.cuda.current_stream(i).cuda_stream without the Stream
# object, which takes longer to make (1.9 us) than everything else a call checks.
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


class LogProb(NamedTuple):
    logp: Optional[torch.Tensor] = None      # [rows] fp32
    entropy: Optional[torch.Tensor] = None   # [rows] fp32
    stats: Optional[torch.Tensor] = None     # [rows, 2] fp32: largest logit, log of the sum relative to it


class PolicyLoss(NamedTuple):
    loss: Optional[torch.Tensor] = None      # [1] fp32
    dlogp: Optional[torch.Tensor] = None     # [B, S] fp32
    dentropy: Optional[torch.Tensor] = None  # [B, S] fp32; None without entropy
    metrics: Optional[torch.Tensor] = None   # [6] fp32: surrogate, KL to ref, entropy, clipped, KL to old, ratio
    counts: Optional[torch.Tensor] = None    # [2] int64: tokens, sequences


class PreferenceLoss(NamedTuple):
    loss: Optional[torch.Tensor] = None       # [1] fp32
    dlogp: Optional[torch.Tensor] = None      # [2 P, S] fp32
    pair_loss: Optional[torch.Tensor] = None  # [P] fp32
    rewards: Optional[torch.Tensor] = None    # [2 P] fp32
    metrics: Optional[torch.Tensor] = None    # [4] fp32: accuracy, reward of the chosen, of the rejected, h
    counts: Optional[torch.Tensor] = None     # [1] int64: pairs


def _require(name, t, dev, dtype, shape):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a tensor, got {type(t).__name__}")
    if t.dtype is not dtype or t.shape != shape or t.device != dev or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {dev}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _rows(name, t, dev=None):
    """(pointer, rows, columns, row stride, is bf16) of a matrix whose rows are contiguous."""
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a tensor, got {type(t).__name__}")
    if t.dim() != 2 or t.dtype not in (_F32, _BF16) or not t.is_cuda or (dev is not None and t.device != dev):
        raise ValueError(f"{name}: expected a float32 or bfloat16 matrix on {dev or 'a GPU'}, got {t.dtype} "
                         f"{tuple(t.shape)} on {t.device}")
    n, c = t.shape
    if (c > 1 and t.stride(1) != 1) or (n > 1 and t.stride(0) < c):
        raise ValueError(f"{name}: rows must be contiguous and not overlap, got strides {t.stride()}")
    return t.data_ptr(), n, c, (t.stride(0) if n > 1 else c), t.dtype == _BF16


def _out(name, t, dev, dtype, shape):
    if t is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    if t.dtype is not dtype or t.shape != shape or t.device != dev or not t.is_contiguous():
        _require("out." + name, t, dev, dtype, torch.Size(shape))
    return t


def _workspace(t, need, dev):
    if t is None:
        if need == 0:
            return None, 0
        t = torch.empty(need, dtype=_U8, device=dev)
    elif t.device != dev or t.dtype != _U8 or not t.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous uint8 tensor on {dev}")
    return t, t.numel()


def _launch(dev, fn, *args):
    """fn(*args, stream) on dev's current stream."""
    if torch.cuda.current_device() == dev.index:
        fn(*args, _stream(dev.index))
    else:
        with torch.cuda.device(dev):
            fn(*args, _stream(dev.index))


def _ptr(t):
    return None if t is None else t.data_ptr()


def _row_outputs(out, n, dev):
    out = out or LogProb()
    return LogProb(_out("logp", out.logp, dev, _F32, (n,)), _out("entropy", out.entropy, dev, _F32, (n,)),
                   _out("stats", out.stats, dev, _F32, (n, 2)))


def token_logprob(logits, targets, *, inv_temperature: float = 1.0, out: Optional[LogProb] = None,
                  workspace=None) -> LogProb:
    """Log-probability of targets[r] (int32; outside the vocabulary: the row is ignored) and entropy of
    every row of logits [rows, vocab] (fp32 or bf16, rows contiguous) times inv_temperature."""
    p, n, v, ld, bf = _rows("logits", logits)
    dev = logits.device
    t = _require("targets", targets, dev, _I32, torch.Size((n,)))
    out = _row_outputs(out, n, dev)
    ws, nb = _workspace(workspace, B.token_logprob_workspace_bytes(n, v), dev)
    _launch(dev, B.token_logprob, n, v, p, ld, bf, t, inv_temperature, out.logp.data_ptr(), out.entropy.data_ptr(),
            out.stats.data_ptr(), _ptr(ws), nb)
    return out


def token_logprob_backward(logits, targets, forward: LogProb, dlogp, dentropy=None, *, inv_temperature: float = 1.0,
                           out=None) -> torch.Tensor:
    """Gradient in the logits, given the forward's outputs and the gradients in its logp and (optional)
    entropy.  out: fp32 or bf16 [rows, vocab], may be the logits; of the logits' type when not given."""
    p, n, v, ld, bf = _rows("logits", logits)
    dev = logits.device
    t = _require("targets", targets, dev, _I32, torch.Size((n,)))
    row = torch.Size((n,))
    s = _require("forward.stats", forward.stats, dev, _F32, torch.Size((n, 2)))
    g = _require("dlogp", dlogp, dev, _F32, row)
    h = e = None
    if dentropy is not None:
        h = _require("dentropy", dentropy, dev, _F32, row)
        e = _require("forward.entropy", forward.entropy, dev, _F32, row)
    if out is None:
        out = torch.empty(n, v, dtype=logits.dtype, device=dev)
    o, on, ov, ldo, obf = _rows("out", out, dev)
    if (on, ov) != (n, v):
        raise ValueError(f"out: expected shape {(n, v)}, got {(on, ov)}")
    _launch(dev, B.token_logprob_backward, n, v, p, ld, bf, t, s, e, g, h, inv_temperature, o, ldo, obf)
    return out


def head_logprob(x, weight, targets, *, inv_temperature: float = 1.0, out: Optional[LogProb] = None,
                 workspace=None) -> LogProb:
    """token_logprob of the logits x weight^T (x [rows, d], weight [vocab, d], both fp32 or both bf16),
    without the logits in memory."""
    px, n, d, ldx, bf = _rows("x", x)
    dev = x.device
    pw, v, dw, ldw, wbf = _rows("weight", weight, dev)
    if d != dw or bf != wbf:
        raise ValueError(f"x {x.dtype} {tuple(x.shape)} and weight {weight.dtype} {tuple(weight.shape)} do not match")
    t = _require("targets", targets, dev, _I32, torch.Size((n,)))
    out = _row_outputs(out, n, dev)
    ws, nb = _workspace(workspace, B.head_logprob_workspace_bytes(n, v, d, bf), dev)
    _launch(dev, B.head_logprob, n, v, d, px, ldx, pw, ldw, bf, t, inv_temperature, out.logp.data_ptr(),
            out.entropy.data_ptr(), out.stats.data_ptr(), _ptr(ws), nb)
    return out


def _mask(mask, dev, shape):
    if getattr(mask, "dtype", None) is torch.bool:
        mask = mask.view(_U8)
    return _require("mask", mask, dev, _U8, shape)


def _grid(name, t):
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: expected a tensor, got {type(t).__name__}")
    if t.dim() != 2 or not t.is_cuda:
        raise ValueError(f"{name}: expected a [sequences, length] tensor on a GPU, got {tuple(t.shape)} on {t.device}")
    return t.device, t.shape


def policy_loss(logp, old_logp, advantages, mask, *, ref_logp=None, entropy=None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, entropy_coef: float = 0.0, reduction: str = "token",
                norm: float = 0.0, grad_scale: float = 1.0, out: Optional[PolicyLoss] = None,
                workspace=None) -> PolicyLoss:
    """Clipped policy loss with a KL term to ref_logp and an entropy bonus, and its gradients in logp and
    entropy.  All [B, S] fp32 (advantages [B] or [B, S]); mask [B, S] bool or uint8, where 0 the other arrays may
    hold anything.  reduction "token": mean over the tokens that count; "sequence": mean over the sequences
    that have any of their means; norm > 0 divides instead of the number of tokens (of sequences)."""
    dev, shape = _grid("logp", logp)
    b, s = shape
    lp = _require("logp", logp, dev, _F32, shape)
    old = _require("old_logp", old_logp, dev, _F32, shape)
    ref = None if ref_logp is None else _require("ref_logp", ref_logp, dev, _F32, shape)
    ent = None if entropy is None else _require("entropy", entropy, dev, _F32, shape)
    per_token = getattr(advantages, "ndim", 1) == 2
    adv = _require("advantages", advantages, dev, _F32, shape if per_token else torch.Size((b,)))
    m = _mask(mask, dev, shape)
    if reduction not in _REDUCTIONS:
        raise ValueError(f"reduction: {reduction!r} is not one of {sorted(_REDUCTIONS)}")
    out = out or PolicyLoss()
    if entropy is None and out.dentropy is not None:
        raise ValueError("out.dentropy needs entropy")
    out = PolicyLoss(_out("loss", out.loss, dev, _F32, (1,)), _out("dlogp", out.dlogp, dev, _F32, (b, s)),
                     None if entropy is None else _out("dentropy", out.dentropy, dev, _F32, (b, s)),
                     _out("metrics", out.metrics, dev, _F32, (6,)), _out("counts", out.counts, dev, torch.int64, (2,)))
    hp = B.PolicyHParams(clip_low, clip_high, kl_coef, entropy_coef, norm, grad_scale, _REDUCTIONS[reduction],
                         per_token)
    ws, nb = _workspace(workspace, B.policy_loss_workspace_bytes(b, s), dev)
    _launch(dev, B.policy_loss, b, s, lp, old, ref, ent, adv, m, hp, out.loss.data_ptr(), out.dlogp.data_ptr(),
            _ptr(out.dentropy), out.metrics.data_ptr(), out.counts.data_ptr(), _ptr(ws), nb)
    return out


def preference_loss(logp, mask, *, ref_logp=None, kind: str = "sigmoid", beta: float = 0.1,
                    label_smoothing: float = 0.0, margin: float = 0.0, length_normalize: bool = False,
                    norm: float = 0.0, grad_scale: float = 1.0, out: Optional[PreferenceLoss] = None,
                    workspace=None) -> PreferenceLoss:
    """Preference loss of P pairs and its gradient in logp.  logp, ref_logp [2 P, S] fp32, the chosen
    answers first, then the rejected ones in the same order; mask [2 P, S] bool or uint8.  kind "sigmoid",
    "hinge" or "square"; pairs with a row of no tokens do not count; norm > 0 divides instead of their number."""
    dev, shape = _grid("logp", logp)
    rows, s = shape
    if rows % 2:
        raise ValueError(f"logp: expected 2 P rows, got {rows}")
    p = rows // 2
    lp = _require("logp", logp, dev, _F32, shape)
    ref = None if ref_logp is None else _require("ref_logp", ref_logp, dev, _F32, shape)
    m = _mask(mask, dev, shape)
    if kind not in _KINDS:
        raise ValueError(f"kind: {kind!r} is not one of {sorted(_KINDS)}")
    out = out or PreferenceLoss()
    out = PreferenceLoss(_out("loss", out.loss, dev, _F32, (1,)), _out("dlogp", out.dlogp, dev, _F32, (rows, s)),
                         _out("pair_loss", out.pair_loss, dev, _F32, (p,)),
                         _out("rewards", out.rewards, dev, _F32, (rows,)),
                         _out("metrics", out.metrics, dev, _F32, (4,)),
                         _out("counts", out.counts, dev, torch.int64, (1,)))
    hp = B.PreferenceHParams(beta, label_smoothing, margin, _KINDS[kind], int(length_normalize), norm, grad_scale)
    ws, nb = _workspace(workspace, B.preference_loss_workspace_bytes(p, s), dev)
    _launch(dev, B.preference_loss, p, s, lp, ref, m, hp, out.loss.data_ptr(), out.dlogp.data_ptr(),
            out.pair_loss.data_ptr(), out.rewards.data_ptr(), out.metrics.data_ptr(), out.counts.data_ptr(),
            _ptr(ws), nb)
    return out
