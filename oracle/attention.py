"""Oracle of attention over key ranges, its key ranges and the counter-based dropout (numpy, any float dtype).

TEST INFRASTRUCTURE: only the tests may use this module.  It shares no code with the HIP path.

Every function is the definition, head by head; gradients are the chain rule, pinned by finite differences."""
from __future__ import annotations

import numpy as np


def key_ranges(ids, prefix=None):
    """(start, end) [B, S]: token by token."""
    B, S = ids.shape
    start, end = np.zeros((B, S), np.int32), np.zeros((B, S), np.int32)
    for b in range(B):
        for i in range(S):
            if ids[b, i] < 0:
                continue
            lo = i
            while lo > 0 and ids[b, lo - 1] == ids[b, i]:
                lo -= 1
            hi = i + 1
            if prefix is not None and prefix[b, lo:i + 1].all():
                while hi < S and ids[b, hi] == ids[b, i] and prefix[b, hi]:
                    hi += 1
            start[b, i], end[b, i] = lo, hi
    return start, end


def causal_ranges(B, Sq, Sk, q_start=None):
    """The ranges of queries at positions q_start[b] + i that see the keys at or before them."""
    first = np.full(B, Sk - Sq) if q_start is None else np.asarray(q_start)
    end = np.clip(first[:, None] + np.arange(Sq)[None, :] + 1, 0, Sk)
    return np.zeros((B, Sq), np.int64), end


def _scores(q, k, b, h, kh, first, scale, cap, slopes):
    """(scores, their derivative in scale q.k, scale sum |q| |k|) of one head"""
    x = scale * q[b, :, h] @ k[b, :, kh].T
    mag = scale * np.abs(q[b, :, h]) @ np.abs(k[b, :, kh]).T
    g = np.ones_like(x)
    if cap:
        t = np.tanh(x / cap)
        x, g = cap * t, 1.0 / np.cosh(x / cap) ** 2
    if slopes is not None:
        far = np.abs((first + np.arange(q.shape[1]))[:, None] - np.arange(k.shape[1])[None, :])
        x = x - slopes[h] * far
    return x, g, mag


def _visible(start, end, b, Sk):
    j = np.arange(Sk)[None, :]
    return (j >= start[b][:, None]) & (j < end[b][:, None])


def attention(q, k, v, start, end, q_start=None, scale=None, cap=0.0, slopes=None):
    """(o [B, Sq, H, hd], lse [B, H, Sq]); values outside a query's range are never touched."""
    B, Sq, H, hd = q.shape
    Sk, KV = k.shape[1], k.shape[2]
    scale = 1.0 / np.sqrt(hd) if scale is None else scale
    o, lse = np.zeros((B, Sq, H, hd)), np.full((B, H, Sq), -np.inf)
    for b in range(B):
        first = Sk - Sq if q_start is None else q_start[b]
        see = _visible(start, end, b, Sk)
        for h in range(H):
            s, _, _ = _scores(q, k, b, h, h // (H // KV), first, scale, cap, slopes)
            for i in range(Sq):
                js = np.nonzero(see[i])[0]
                if js.size == 0:
                    continue
                m = s[i, js].max()
                e = np.exp(s[i, js] - (0.0 if m == -np.inf else m))
                lse[b, h, i] = (0.0 if m == -np.inf else m) + (np.log(e.sum()) if e.sum() else -np.inf)
                o[b, i, h] = (e / e.sum()) @ v[b, js, h // (H // KV)] if e.sum() else 0.0
    return o, lse


def attention_bwd(q, k, v, dout, start, end, q_start=None, scale=None, cap=0.0, slopes=None, errors=None):
    """(dq, dk, dv).  With errors = (score, prob, grad, delta): also bounds of what relative errors `prob` of every
    P entry, `grad` of every dS entry, an error `score` (1 + sum |q||k| scale + |s|) of every score and one `delta`
    sum |dO| |o| of every delta make of the three (each summed without cancellation)."""
    B, Sq, H, hd = q.shape
    Sk, KV = k.shape[1], k.shape[2]
    scale = 1.0 / np.sqrt(hd) if scale is None else scale
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    bq, bk, bv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(B):
        first = Sk - Sq if q_start is None else q_start[b]
        see = _visible(start, end, b, Sk)
        rows = np.nonzero(see.any(1))[0]
        cols = np.nonzero(see.any(0))[0]
        if rows.size == 0:
            continue
        sub = see[np.ix_(rows, cols)]
        for h in range(H):
            kh = h // (H // KV)
            qs, ks, vs, ds_ = q[b, rows, h], k[b, cols, kh], v[b, cols, kh], dout[b, rows, h]
            s, g, mag = _scores(q, k, b, h, kh, first, scale, cap, slopes)
            s, g, mag = s[np.ix_(rows, cols)], g[np.ix_(rows, cols)], mag[np.ix_(rows, cols)]
            s = np.where(sub, s, -np.inf)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            dp = ds_ @ vs.T
            delta = (p * dp).sum(1, keepdims=True)
            dz = p * (dp - delta) * g
            dq[b, rows, h] = scale * dz @ ks
            dk[b, cols, kh] += scale * dz.T @ qs
            dv[b, cols, kh] += p.T @ ds_
            if errors is not None:
                score, prob, grad, dl = errors
                es = np.where(sub, score * (1 + mag + np.abs(np.where(sub, s, 0.0))), 0.0)
                ep = es + es.max(1, keepdims=True) + prob
                adp = np.abs(ds_) @ np.abs(vs).T
                eds = (p * g * (np.abs(dp - delta) * (ep + grad) + score * adp
                                + dl * (np.abs(ds_) * (p @ np.abs(vs))).sum(1, keepdims=True)) + score * p * np.abs(dp - delta))
                bq[b, rows, h] = scale * eds @ np.abs(ks)
                bk[b, cols, kh] += scale * eds.T @ np.abs(qs)
                bv[b, cols, kh] += (p * ep).T @ np.abs(ds_)
    return (dq, dk, dv) if errors is None else (dq, dk, dv, bq, bk, bv)


def attention_bounds(q, k, v, start, end, score, prob, q_start=None, scale=None, cap=0.0, slopes=None):
    """Bounds of the errors of o and lse for an error score (1 + sum |q||k| scale + |s|) of every score and a relative
    one `prob` of every probability."""
    B, Sq, H, hd = q.shape
    Sk, KV = k.shape[1], k.shape[2]
    scale = 1.0 / np.sqrt(hd) if scale is None else scale
    bo, bl = np.zeros((B, Sq, H, hd)), np.zeros((B, H, Sq))
    for b in range(B):
        first = Sk - Sq if q_start is None else q_start[b]
        see = _visible(start, end, b, Sk)
        for h in range(H):
            kh = h // (H // KV)
            s, _, mag = _scores(q, k, b, h, kh, first, scale, cap, slopes)
            for i in range(Sq):
                js = np.nonzero(see[i])[0]
                if js.size == 0:
                    continue
                si = s[i, js]
                p = np.exp(si - si.max())
                p /= p.sum()
                es = score * (1 + mag[i, js] + np.abs(si))
                bl[b, h, i] = es.max()
                bo[b, i, h] = (p * (es + es.max() + prob)) @ np.abs(v[b, js, kh])
    return bo, bl


def philox(counter, key):
    """Philox4x32-10 of one counter (4 words) and key (2 words), in Python integers."""
    x, (k0, k1) = list(counter), key
    for _ in range(10):
        a, b = 0xD2511F53 * x[0], 0xCD9E8D57 * x[2]
        x = [(b >> 32) ^ x[1] ^ k0, b & 0xFFFFFFFF, (a >> 32) ^ x[3] ^ k1, a & 0xFFFFFFFF]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return x


def dropout_keep(rows, cols, p, seed, offset):
    """The kept elements [rows, cols] (truth values) and the factor of what is kept."""
    t = round(p * 65536)
    u = []
    for g in range((rows * cols + 7) // 8):
        for w in philox((g & 0xFFFFFFFF, g >> 32, offset & 0xFFFFFFFF, offset >> 32), (seed & 0xFFFFFFFF, seed >> 32)):
            u += [w & 0xFFFF, w >> 16]
    return np.array(u[:rows * cols]).reshape(rows, cols) >= t, 65536.0 / (65536 - t)
