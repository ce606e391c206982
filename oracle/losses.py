"""Oracle of the log-probability operators and the losses on them (numpy, any float dtype).

TEST INFRASTRUCTURE: only the tests may use this module.  It shares no code with the HIP path.

Every function is the textbook definition; gradients are the chain rule of the matching forward, pinned by
finite differences in the tests."""
from __future__ import annotations

import numpy as np


# ---------------------------------------------------------------- rows of logits
def token_logprob(x, targets, s):
    """(logp, entropy, stats) of rows x [T, V] times s; targets outside [0, V) are ignored (zeros)."""
    T, V = x.shape
    logp, ent, stats = np.zeros(T, x.dtype), np.zeros(T, x.dtype), np.zeros((T, 2), x.dtype)
    for r in range(T):
        t = int(targets[r])
        if not 0 <= t < V:
            continue
        m = np.max(x[r])
        if m == -np.inf:
            logp[r], stats[r] = -np.inf, (-np.inf, 0.0)
            continue
        with np.errstate(invalid="ignore"):  # +inf among the logits
            z = s * (x[r] - m)
            e = np.exp(z)
            logs = np.log(e.sum())
            logp[r] = z[t] - logs
            ent[r] = logs - np.sum(np.where(e > 0, e * np.where(e > 0, z, 0.0), e)) / e.sum()
        stats[r] = (m, logs)
    return logp, ent, stats


def token_logprob_bwd(x, targets, s, g, h=None):
    """d(sum g logp + h entropy)/dx."""
    T, V = x.shape
    dx = np.zeros_like(x)
    for r in range(T):
        t = int(targets[r])
        m = np.max(x[r])
        hr = 0.0 if h is None else h[r]
        if not 0 <= t < V or m == -np.inf or (g[r] == 0 and hr == 0):
            continue
        with np.errstate(invalid="ignore"):
            z = s * (x[r] - m)
        lp = z - np.log(np.exp(z).sum())
        p = np.exp(lp)
        lp0 = np.where(p > 0, lp, 0.0)
        H = -np.sum(p * lp0)
        one = np.zeros(V, x.dtype)
        one[t] = 1.0
        dx[r] = s * (g[r] * (one - p) - hr * p * (lp0 + H))
    return dx


# ---------------------------------------------------------------- policy loss
def _kl(d):
    """e^d - 1 - d, infinite at both ends"""
    return np.inf if np.isinf(d) else np.expm1(d) - d


def policy_loss(logp, old, adv, mask, *, ref=None, entropy=None, clip_low=0.2, clip_high=0.2, kl_coef=0.0,
                entropy_coef=0.0, reduction="token", norm=0.0, grad_scale=1.0):
    """dict of loss, dlogp, dentropy, metrics [6], counts [2]; [B, S] arrays, adv [B] or [B, S]."""
    B, S = logp.shape
    on = mask != 0
    n = on.sum(1)
    tokens, seqs = int(n.sum()), int((n > 0).sum())
    dlogp, dent, met = np.zeros((B, S)), np.zeros((B, S)), np.zeros(6)
    for b in range(B):
        for t in np.nonzero(on[b])[0]:
            if reduction == "sequence":
                w = 1.0 / ((norm if norm > 0 else seqs) * n[b])
            else:
                w = 1.0 / (norm if norm > 0 else tokens)
            a = float(adv[b, t] if adv.ndim == 2 else adv[b])
            x = float(logp[b, t]) - float(old[b, t])
            r = np.exp(x)
            cut = (a > 0 and x > np.log1p(clip_high)) or (a < 0 and x < np.log1p(-clip_low))
            met[0] += w * max(-r * a, -min(max(r, 1.0 - clip_low), 1.0 + clip_high) * a)
            met[3] += w * cut
            met[4] += w * _kl(x)
            met[5] += w * r
            g = 0.0 if cut else -r * a
            if ref is not None:
                d = float(ref[b, t]) - float(logp[b, t])
                met[1] += w * _kl(d)
                g -= kl_coef * np.expm1(d) if kl_coef else 0.0
            if entropy is not None:
                met[2] += w * float(entropy[b, t])
            dlogp[b, t] = grad_scale * w * g
            dent[b, t] = -grad_scale * w * entropy_coef
    # a term without a weight adds nothing, also where it is infinite
    loss = met[0] + (kl_coef * met[1] if kl_coef else 0.0) - (entropy_coef * met[2] if entropy_coef else 0.0)
    return dict(loss=loss, dlogp=dlogp,
                dentropy=dent if entropy is not None else None, metrics=met, counts=np.array([tokens, seqs]))


# ---------------------------------------------------------------- preference loss
def preference_loss(logp, mask, *, ref=None, kind="sigmoid", beta=0.1, label_smoothing=0.0, margin=0.0,
                    length_normalize=False, norm=0.0, grad_scale=1.0):
    """dict of loss, dlogp, pair_loss [P], rewards [2 P], metrics [4], counts [1]; rows chosen, then rejected."""
    P = logp.shape[0] // 2
    on = mask != 0
    n = on.sum(1)
    v = np.where(on, logp, 0.0)
    if ref is not None:
        v = v - np.where(on, ref, 0.0)
    score = np.array([v[i][on[i]].sum() for i in range(2 * P)])
    if length_normalize:
        score = score / np.maximum(n, 1)
    dlogp, pair, rewards, met = np.zeros(logp.shape), np.zeros(P), np.zeros(2 * P), np.zeros(4)
    live = [p for p in range(P) if n[p] > 0 and n[p + P] > 0]
    den = norm if norm > 0 else max(1, len(live))
    for p in live:
        delta = score[p] - score[p + P]
        h = beta * delta - margin
        if kind == "sigmoid":
            ls = lambda u: -np.logaddexp(0.0, -u)  # noqa: E731
            pair[p] = -(1.0 - label_smoothing) * ls(h) - label_smoothing * ls(-h)
            dh = -(1.0 - label_smoothing) * np.exp(ls(-h)) + label_smoothing * np.exp(ls(h))
        elif kind == "hinge":
            pair[p] = max(0.0, 1.0 - h)
            dh = -1.0 if h < 1.0 else 0.0
        else:
            pair[p] = ((h - 0.5) / beta) ** 2
            dh = 2.0 * (h - 0.5) / beta ** 2
        rewards[p], rewards[p + P] = beta * score[p], beta * score[p + P]
        met += np.array([float(delta > 0), rewards[p], rewards[p + P], h]) / den
        for row, sign in ((p, 1.0), (p + P, -1.0)):
            c = grad_scale * sign * beta * dh / den
            dlogp[row, on[row]] = c / n[row] if length_normalize else c
    return dict(loss=pair.sum() / den, dlogp=dlogp, pair_loss=pair, rewards=rewards, metrics=met,
                counts=np.array([len(live)]))
