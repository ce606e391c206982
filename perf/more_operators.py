"""Speed cases of the operators that train and run blocks on packed documents.

  ranges     attention.key_ranges: from the documents (and prefixes) packed in a row, the keys that each query sees
  attn       attention.attention: softmax attention over those keys, its scores capped by a tanh or lowered by the
             distance between query and key; a few queries against a long cache as well as whole rows
  attn_grad  attention.attention_backward: its gradients in queries, keys and values
  dropout    dropout.dropout_add (and dropout_backward): a counter-based mask that is never stored, with the residual

listed() names the cases, draw(rng) gives more of the same ranges.  run() is the plain form of an operator
(elementary torch operations) or, where `own` is true, the call a user makes of the package.  exact() is
the definition in float64.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEV = "cuda:0"


# ------------------------------------------------------------------------------------------ cases
def _attn(op, batch, q, k, heads, kv, hd, f32=False, docs=0, prefix=False, cap=0.0, bias=False, keep=False, ragged=False):
    return dict(op=op, batch=batch, q=q, k=k, heads=heads, kv=kv, hd=hd, f32=f32, docs=docs, prefix=prefix, cap=cap,
                bias=bias, keep=keep, ragged=ragged)


def _ranges(batch, length, docs, prefix):
    return dict(op="ranges", batch=batch, length=length, docs=docs, prefix=prefix)


def _drop(rows, d, p, f32=False, residual=True, pad=0):
    return dict(op="dropout", rows=rows, d=d, p=p, f32=f32, residual=residual, pad=pad)


def listed():
    return [
        # one new token of one answer against the 2048 before it: latency
        dict(_attn("attn", 1, 1, 2048, 16, 16, 128, cap=50.0), name="attn-one-token"),
        # one new token of each of 16 answers of different lengths up to 32768: the cache is read once
        dict(_attn("attn", 16, 1, 32768, 32, 8, 128, bias=True, ragged=True), name="attn-long-cache"),
        # a block's training forward on packed documents (4 x 2048 tokens, 16 heads of 128)
        dict(_attn("attn", 4, 2048, 2048, 16, 16, 128, docs=6, keep=True), name="attn-documents"),
        # two rows of 4096 tokens, capped scores, a few documents a row
        dict(_attn("attn", 2, 4096, 4096, 32, 8, 128, docs=3, cap=50.0, keep=True), name="attn-large"),
        # an fp32 stage, odd lengths, prompts that see themselves whole, a distance bias
        dict(_attn("attn", 3, 777, 777, 12, 4, 64, f32=True, docs=4, prefix=True, bias=True), name="attn-odd-f32"),
        # the backward of a small block: 8 x 1024 tokens, 12 heads of 64, packed
        dict(_attn("attn_grad", 8, 1024, 1024, 12, 12, 64, docs=5), name="grad-small"),
        # the backward of attn-large
        dict(_attn("attn_grad", 2, 4096, 4096, 32, 8, 128, docs=3, cap=50.0), name="grad-large"),
        # the smallest heads in fp32, odd length, prefixes and a bias
        dict(_attn("attn_grad", 2, 333, 333, 8, 2, 32, f32=True, docs=3, prefix=True, bias=True), name="grad-odd-f32"),
        # the ranges of one microbatch
        dict(_ranges(8, 1024, 5, False), name="ranges-batch"),
        # few long rows of many answers behind their prompts
        dict(_ranges(4, 131072, 200, True), name="ranges-long"),
        # an odd number of short rows, fp32: latency
        dict(_drop(37, 515, 0.1, f32=True), name="dropout-few"),
        # a branch's output of 8192 tokens added to the residual stream
        dict(_drop(8192, 4096, 0.1), name="dropout-large"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ranges", "attn", "attn", "attn_grad", "attn_grad", "dropout"])
    if op == "ranges":
        length = _log(rng, 1, 131072)
        return _ranges(_log(rng, 1, max(1, min(256, 5.0e5 / length))), length, _log(rng, 1, 200), rng.random() < 0.5)
    if op == "dropout":
        d = _log(rng, 1, 8192)
        return _drop(_log(rng, 1, max(1, min(65536, 3.3e7 / d))), d, rng.choice([0.0, 0.05, 0.1, 0.5]), rng.random() < 0.4,
                     rng.random() < 0.6, rng.choice([0, 0, 8, 3]))
    f32 = rng.random() < 0.25
    hd = rng.choice([32, 64, 128])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 1, 2, 4, 8])
    cap, bias = rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.4
    slow = f32 or hd == 32
    if op == "attn" and rng.random() < 0.4:  # a few queries against a cache
        q = _log(rng, 1, 16)
        k = max(q, _log(rng, 1, 32768))
        batch = _log(rng, 1, max(1, min(64, (1.2e8 if slow else 5.0e8) / (k * kv * hd))))
        return _attn(op, batch, q, k, heads, kv, hd, f32, cap=cap, bias=bias, ragged=rng.random() < 0.5)
    s = _log(rng, 1, 4096)
    batch = _log(rng, 1, max(1, min(16, (1.0e10 if slow else 1.2e11) / (heads * hd * float(s) * s))))
    if slow and heads * hd * float(s) * s * batch > 2.0e10:
        s = int(math.sqrt(2.0e10 / (heads * hd * batch)))
    return _attn(op, batch, s, s, heads, kv, hd, f32, docs=rng.choice([0, 1, 3, 8]), prefix=rng.random() < 0.3, cap=cap,
                 bias=bias, keep=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _lengths(length, docs):
    """The lengths of a row's documents and, last, of its padding: the same for every seed, which orders them."""
    rng = random.Random(length * 1009 + docs)
    w = [0.2 + rng.random() for _ in range(docs)]
    pad = length // 32 if docs > 1 else 0
    out = [int((length - pad) * x / sum(w)) for x in w]
    out[0] += length - pad - sum(out)
    return out, pad


def _prefix_of(n):
    return n // 3


def _documents(batch, length, docs, seed):
    """Document ids [batch, length] (padding -1 behind them) and the flags of the tokens of a document's prefix."""
    rng = random.Random(seed * 7919 + 13)
    lens, pad = _lengths(length, docs)
    ids, flags = np.full((batch, length), -1, np.int32), np.zeros((batch, length), np.uint8)
    for b in range(batch):
        order = list(range(docs))
        rng.shuffle(order)
        at = 0
        for n, which in enumerate(order):
            ids[b, at:at + lens[which]] = n
            flags[b, at:at + _prefix_of(lens[which])] = 1
            at += lens[which]
    return torch.from_numpy(ids).to(DEV), torch.from_numpy(flags).to(DEV)


def _cache_lengths(case):
    """The answers' lengths so far, the longest filling the cache."""
    rng = random.Random(case["k"] * 31 + case["batch"])
    out = [case["q"] + int((case["k"] - case["q"]) * rng.random()) for _ in range(case["batch"])]
    out[0] = case["k"]
    return out


def _slopes(n):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / n) for h in range(n)], dtype=torch.float32, device=DEV)


def _attn_inputs(c, seed):
    g = _gen(seed)
    dt = torch.float32 if c["f32"] else torch.bfloat16
    norm = lambda n, heads, std: torch.empty(c["batch"], n, heads, c["hd"], dtype=dt, device=DEV).normal_(0.0, std, generator=g)  # noqa: E731
    s = dict(case=c, q=norm(c["q"], c["heads"], 3.0 if c["cap"] else 1.0), k=norm(c["k"], c["kv"], 1.0),
             v=norm(c["k"], c["kv"], 1.0), slopes=_slopes(c["heads"]) if c["bias"] else None, start=None, end=None,
             q_start=None, scale=1.0 / math.sqrt(c["hd"]), cap=c["cap"])
    if c["docs"]:
        ids, flags = _documents(c["batch"], c["k"], c["docs"], seed)
        s["start"], s["end"] = _plain_ranges(ids, flags if c["prefix"] else None)
    if c["ragged"]:
        lens = _cache_lengths(c)
        random.Random(seed).shuffle(lens)
        s["q_start"] = torch.tensor(lens, dtype=torch.int32, device=DEV) - c["q"]
    return s, g


def prepare(case, seed):
    c = case
    if c["op"] == "ranges":
        ids, flags = _documents(c["batch"], c["length"], c["docs"], seed)
        i32 = dict(dtype=torch.int32, device=DEV)
        return dict(case=c, ids=ids, flags=flags if c["prefix"] else None,
                    out=(torch.empty(c["batch"], c["length"], **i32), torch.empty(c["batch"], c["length"], **i32)))
    if c["op"] == "dropout":
        g = _gen(seed)
        dt = torch.float32 if c["f32"] else torch.bfloat16
        new = lambda: torch.empty(c["rows"], c["d"] + c["pad"], dtype=dt, device=DEV).normal_(0.0, 1.0, generator=g)[:, :c["d"]]  # noqa: E731
        rng = random.Random(seed)
        return dict(case=c, x=new(), residual=new() if c["residual"] else None, seed=rng.getrandbits(64),
                    offset=rng.getrandbits(40), out=torch.empty(c["rows"], c["d"], dtype=dt, device=DEV))
    s, g = _attn_inputs(c, seed)
    n = (c["batch"], c["q"], c["heads"], c["hd"])
    dt = s["q"].dtype
    if c["op"] == "attn":
        s["out"] = dict(o=torch.empty(n, dtype=dt, device=DEV),
                        lse=torch.empty(c["batch"], c["heads"], c["q"], device=DEV),
                        o_f32=torch.empty(n, device=DEV) if c["keep"] and not c["f32"] else None)
        return s
    # what the forward left, and a gradient of the output
    fwd = _plain_attention(s)
    s.update(o=fwd["o_f32"].to(dt), lse=fwd["lse"], o_f32=None if c["f32"] else fwd["o_f32"],
             dout=torch.empty(n, dtype=dt, device=DEV).normal_(0.0, 1.0, generator=g),
             grads=(torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["v"])))
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_ranges(ids, flags):
    b, n = ids.shape
    at = torch.arange(n, dtype=torch.int32, device=DEV).expand(b, n)
    live = ids >= 0
    new = torch.ones_like(live)
    new[:, 1:] = ids[:, 1:] != ids[:, :-1]
    zero = torch.zeros_like(at)
    start = torch.where(new, at, zero).cummax(1).values
    end = at + 1
    if flags is not None:
        plain = flags == 0
        inside = torch.where(plain, at, zero - 1).cummax(1).values < start
        stop = torch.where(new | plain, at, zero + n)  # where a prefix that began earlier ends
        stop = torch.cat([stop, torch.full((b, 1), n, dtype=torch.int32, device=DEV)], 1)
        stop = stop.flip(1).cummin(1).values.flip(1)[:, 1:]
        end = torch.where(inside, stop, end)
    return torch.where(live, start, zero).contiguous(), torch.where(live, end, zero).contiguous()


def _grouped(x, kv):
    """[B, S, H, hd] -> [B, kv, H / kv, S, hd] in 32 bits."""
    b, s, h, d = x.shape
    return x.float().view(b, s, kv, h // kv, d).permute(0, 2, 3, 1, 4).contiguous()


def _plain_scores(s):
    """Scores [B, kv, group, Sq, Sk], the slope of their cap (or None) and what each query sees [B, 1, 1, Sq, Sk]."""
    c = s["case"]
    b, nq, nk, kv, grp = c["batch"], c["q"], c["k"], c["kv"], c["heads"] // c["kv"]
    k = _grouped(s["k"], kv)[:, :, 0]
    x = torch.matmul(_grouped(s["q"], kv).view(b, kv, grp * nq, -1), k.transpose(2, 3).contiguous())
    x = x.view(b, kv, grp, nq, nk) * s["scale"]
    slope = None
    if c["cap"]:
        t = torch.tanh(x / s["cap"])
        x, slope = t * s["cap"], 1.0 - t * t
    first = torch.full((b,), nk - nq, dtype=torch.int32, device=DEV) if s["q_start"] is None else s["q_start"]
    i = first[:, None] + torch.arange(nq, dtype=torch.int32, device=DEV)
    j = torch.arange(nk, dtype=torch.int32, device=DEV)
    if s["slopes"] is not None:
        far = (i[:, :, None] - j).abs().float()[:, None, None]
        x = x - s["slopes"].view(1, kv, grp, 1, 1) * far
    if s["start"] is None:
        see = j <= i[:, :, None]
    else:
        see = (j >= s["start"][:, :, None]) & (j < s["end"][:, :, None])
    return x, slope, see[:, None, None]


def _plain_attention(s):
    c = s["case"]
    b, nq, kv, grp, hd = c["batch"], c["q"], c["kv"], c["heads"] // c["kv"], c["hd"]
    x, _, see = _plain_scores(s)
    x = torch.where(see, x, -math.inf)
    m = x.amax(4, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = torch.exp(x - m)
    total = p.sum(4, keepdim=True)
    lse = (torch.log(total) + m).view(b, c["heads"], nq)
    p = p / torch.where(total == 0.0, 1.0, total)
    o = torch.matmul(p.view(b, kv, grp * nq, -1), _grouped(s["v"], kv)[:, :, 0]).view(b, kv, grp, nq, hd)
    return dict(o_f32=o.permute(0, 3, 1, 2, 4).reshape(b, nq, c["heads"], hd), lse=lse)


def _plain_grad(s):
    c = s["case"]
    b, nq, nk, kv, grp, hd = c["batch"], c["q"], c["k"], c["kv"], c["heads"] // c["kv"], c["hd"]
    x, slope, see = _plain_scores(s)
    lse = s["lse"].view(b, kv, grp, nq, 1)
    p = torch.where(see, torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)), 0.0)
    del x
    do, q = _grouped(s["dout"], kv).view(b, kv, grp * nq, hd), _grouped(s["q"], kv).view(b, kv, grp * nq, hd)
    k, v = _grouped(s["k"], kv)[:, :, 0], _grouped(s["v"], kv)[:, :, 0]
    dp = torch.matmul(do, v.transpose(2, 3).contiguous()).view(b, kv, grp, nq, nk)
    ds = p * (dp - (p * dp).sum(4, keepdim=True))
    del dp
    if slope is not None:
        ds = ds * slope
    ds = ds.view(b, kv, grp * nq, nk)
    dq = torch.matmul(ds, k) * s["scale"]
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q) * s["scale"]
    dv = torch.matmul(p.view(b, kv, grp * nq, nk).transpose(2, 3).contiguous(), do)
    dt = s["q"].dtype
    return dict(dq=dq.view(b, kv, grp, nq, hd).permute(0, 3, 1, 2, 4).reshape(b, nq, c["heads"], hd).to(dt),
                dk=dk.transpose(1, 2).contiguous().to(dt), dv=dv.transpose(1, 2).contiguous().to(dt))


def _wide(a, m):
    """High and low 32 bits of a m, both below 2^32, in int64."""
    low = (a & 0xFFFF) * m
    mid = (a >> 16) * m + (low >> 16)
    return mid >> 16, ((mid & 0xFFFF) << 16) | (low & 0xFFFF)


def _philox(g, offset, seed):
    """Philox4x32-10 of the counters (g, offset) under the key seed: [n, 4] in int64."""
    full = lambda v: torch.full_like(g, v & 0xFFFFFFFF)  # noqa: E731
    x0, x1, x2, x3 = g & 0xFFFFFFFF, g >> 32, full(offset), full(offset >> 32)
    k0, k1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    h0, l0 = _wide(x0, 0xD2511F53)
    h1, l1 = _wide(x2, 0xCD9E8D57)
    for _ in range(9):
        x0, x1, x2, x3 = h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
        h0, l0 = _wide(x0, 0xD2511F53)
        h1, l1 = _wide(x2, 0xCD9E8D57)
    return torch.stack([h1 ^ x1 ^ k0, l1, h0 ^ x3 ^ k1, l0], 1)


def _plain_dropout(s):
    c = s["case"]
    n = c["rows"] * c["d"]
    w = _philox(torch.arange((n + 7) // 8, device=DEV), s["offset"], s["seed"])
    u = torch.stack([w & 0xFFFF, w >> 16], 2).view(-1)[:n].view(c["rows"], c["d"])
    t = round(c["p"] * 65536)
    y = torch.where(u >= t, s["x"].float() * (65536.0 / (65536 - t)), 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


# ------------------------------------------------------------------------------------------ run
def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] == "ranges":
            return _plain_ranges(s["ids"], s["flags"])
        if c["op"] == "attn":
            f = _plain_attention(s)
            out = dict(o=f["o_f32"].to(s["q"].dtype), lse=f["lse"])
            if s["out"]["o_f32"] is not None:
                out["o_f32"] = f["o_f32"]
            return out
        if c["op"] == "attn_grad":
            return _plain_grad(s)
        return dict(y=_plain_dropout(s))
    if c["op"] == "dropout":
        from paper_2606_30634_amd import dropout
        if s["residual"] is None:
            dropout.dropout_backward(s["x"], c["p"], s["seed"], s["offset"], out=s["out"])
        else:
            dropout.dropout_add(s["x"], s["residual"], c["p"], s["seed"], s["offset"], out=s["out"])
        return dict(y=s["out"])
    from paper_2606_30634_amd import attention
    if c["op"] == "ranges":
        attention.key_ranges(s["ids"], prefix=s["flags"], out=s["out"])
        return s["out"]
    how = dict(key_start=s["start"], key_end=s["end"], q_start=s["q_start"], scale=s["scale"], softcap=s["cap"],
               slopes=s["slopes"])
    if c["op"] == "attn":
        out = s["out"]
        attention.attention(s["q"], s["k"], s["v"], keep_f32=out["o_f32"] is not None, out=attention.Attention(**out), **how)
        return {k: v for k, v in out.items() if v is not None}
    fwd = attention.Attention(s["o"], s["lse"], s["o_f32"])
    dq, dk, dv = attention.attention_backward(s["q"], s["k"], s["v"], fwd, s["dout"], out=s["grads"], **how)
    return dict(dq=dq, dk=dk, dv=dv)


# ------------------------------------------------------------------------------------------ work
def _pairs(c):
    """Query-key pairs of one head over the batch."""
    if c["docs"]:
        n = 0
        for x in _lengths(c["k"], c["docs"])[0]:
            p = _prefix_of(x) if c["prefix"] else 0
            n += x * (x + 1) // 2 + p * (p - 1) // 2
        return n * c["batch"]
    if c["ragged"]:
        return sum(c["q"] * (n - c["q"]) + c["q"] * (c["q"] + 1) // 2 for n in _cache_lengths(c))
    return c["batch"] * (c["q"] * (c["k"] - c["q"]) + c["q"] * (c["q"] + 1) // 2)


def work(case):
    c = case
    e = 4 if c.get("f32") else 2
    if c["op"] == "ranges":
        n = c["batch"] * c["length"]
        return dict(bytes=n * (12 + c["prefix"]), flops=4 * n)
    if c["op"] == "dropout":
        n = c["rows"] * c["d"]
        return dict(bytes=n * e * (2 + c["residual"]), flops=12 * n)
    q = c["batch"] * c["q"] * c["heads"] * c["hd"]
    keys = sum(_cache_lengths(c)) if c["ragged"] else c["batch"] * c["k"]
    kv = 2 * keys * c["kv"] * c["hd"]
    rows = c["batch"] * c["q"] * c["heads"] * 4 + (8 * c["batch"] * c["q"] if c["docs"] else 0)
    flops = _pairs(c) * c["heads"] * c["hd"]
    if c["op"] == "attn":
        return dict(bytes=(2 * q + kv) * e + rows + (4 * q if c["keep"] and not c["f32"] else 0), flops=4 * flops)
    # q, dout and the output in fp32 read, dq written; k and v read, dk and dv written
    return dict(bytes=3 * q * e + 4 * q + 2 * kv * e + rows, flops=10 * flops)


# ------------------------------------------------------------------------------------------ exact
def _exact_ranges(ids, flags):
    ids = ids.cpu().numpy()
    flags = np.zeros(ids.shape, np.uint8) if flags is None else flags.cpu().numpy()
    start, end = np.zeros(ids.shape, np.int32), np.zeros(ids.shape, np.int32)
    for b in range(ids.shape[0]):
        row = ids[b]
        cuts = [0, *(np.nonzero(np.diff(row))[0] + 1).tolist(), row.size]
        for lo, hi in zip(cuts[:-1], cuts[1:]):
            if row[lo] < 0:
                continue
            start[b, lo:hi] = lo
            end[b, lo:hi] = np.arange(lo, hi) + 1
            off = np.nonzero(flags[b, lo:hi] == 0)[0]
            end[b, lo:lo + (off[0] if off.size else hi - lo)] = lo + off[0] if off.size else hi
    return torch.from_numpy(start).to(DEV), torch.from_numpy(end).to(DEV)


def _exact_head(s, b, h):
    """Scores of one head in 64 bits, its masked softmax and log-sum, and the inputs."""
    c = s["case"]
    kh = h // (c["heads"] // c["kv"])
    q, k, v = s["q"][b, :, h].double(), s["k"][b, :, kh].double(), s["v"][b, :, kh].double()
    z = (q @ k.t()) * s["scale"]
    raw = z
    if c["cap"]:
        z = s["cap"] * torch.tanh(z / s["cap"])
    row = torch.arange(c["q"], device=DEV)[:, None] + (c["k"] - c["q"] if s["q_start"] is None else s["q_start"][b].long())
    col = torch.arange(c["k"], device=DEV)[None, :]
    if s["slopes"] is not None:
        z = z - s["slopes"][h].double() * (row - col).abs()
    if s["start"] is None:
        hide = col > row
    else:
        hide = (col < s["start"][b][:, None]) | (col >= s["end"][b][:, None])
    z = z.masked_fill(hide, -math.inf)
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse.masked_fill(lse == -math.inf, 0.0)[:, None])
    return q, k, v, raw, p, lse, kh


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["op"] == "ranges":
        return _exact_ranges(s["ids"], s["flags"])
    if c["op"] == "dropout":
        n = c["rows"] * c["d"]
        u = np.empty((n + 7) // 8 * 8, np.uint64)
        m32 = np.uint64(0xFFFFFFFF)
        g = np.arange((n + 7) // 8, dtype=np.uint64)
        word = [g & m32, g >> np.uint64(32), np.full_like(g, s["offset"] & 0xFFFFFFFF), np.full_like(g, s["offset"] >> 32)]
        key = [s["seed"] & 0xFFFFFFFF, s["seed"] >> 32]
        for _ in range(10):
            a, b = word[0] * np.uint64(0xD2511F53), word[2] * np.uint64(0xCD9E8D57)
            word = [(b >> np.uint64(32)) ^ word[1] ^ np.uint64(key[0]), b & m32,
                    (a >> np.uint64(32)) ^ word[3] ^ np.uint64(key[1]), a & m32]
            key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
        for k in range(4):
            u[2 * k::8], u[2 * k + 1::8] = word[k] & np.uint64(0xFFFF), word[k] >> np.uint64(16)
        t = round(c["p"] * 65536)
        keep = torch.from_numpy((u[:n] >= t).reshape(c["rows"], c["d"])).to(DEV)
        y = s["x"].double() * 65536.0 / (65536 - t) * keep
        return dict(y=y if s["residual"] is None else y + s["residual"].double())
    zeros = lambda n, heads: torch.zeros(c["batch"], n, heads, c["hd"], dtype=torch.float64, device=DEV)  # noqa: E731
    if c["op"] == "attn":
        o, lse = zeros(c["q"], c["heads"]), torch.zeros(c["batch"], c["heads"], c["q"], dtype=torch.float64, device=DEV)
        for b in range(c["batch"]):
            for h in range(c["heads"]):
                _, _, v, _, p, lse[b, h], _ = _exact_head(s, b, h)
                o[b, :, h] = p @ v
        out = dict(o=o, lse=lse)
        if s["out"]["o_f32"] is not None:
            out["o_f32"] = o
        return out
    dq, dk, dv = zeros(c["q"], c["heads"]), zeros(c["k"], c["kv"]), zeros(c["k"], c["kv"])
    for b in range(c["batch"]):
        for h in range(c["heads"]):
            q, k, v, raw, p, _, kh = _exact_head(s, b, h)
            do = s["dout"][b, :, h].double()
            dp = do @ v.t()
            dz = p * (dp - (p @ v * do).sum(1, keepdim=True))
            if c["cap"]:
                dz = dz / torch.cosh(raw / s["cap"]) ** 2
            dq[b, :, h] = dz @ k * s["scale"]
            dk[b, :, kh] += dz.t() @ q * s["scale"]
            dv[b, :, kh] += p.t() @ do
    return dict(dq=dq, dk=dk, dv=dv)
