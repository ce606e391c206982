"""Speed cases of the operators between a last stage's logits and a loss on log-probabilities.

  logprob       token_logprob: per row of logits the target's log-probability, the entropy and the row's
                maximum logit and log-sum
  logprob_grad  token_logprob_backward: the gradient of those log-probabilities and entropies in the logits
  head          head_logprob: the same as logprob from hidden states and the head's matrix
  policy        policy_loss: the clipped surrogate with a KL term and an entropy bonus, and its gradients
  preference    preference_loss: the loss of paired log ratios and its gradient

listed() names the cases, draw(rng) gives more of the same ranges.  run() is the plain form of an operator
(elementary torch operations) or, where `own` is true, the call a user makes of the package.  exact() is
the definition in float64, with torch's autograd for the gradients.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"


def _f32(v):
    """The float32 a C caller passes for v."""
    return float(torch.tensor(v, dtype=torch.float32))


# ------------------------------------------------------------------------------------------ cases
def _rows(op, rows, vocab, pad=0, f32=True, inv_temp=1.0, ignored=0.0, **kw):
    return dict(op=op, rows=rows, vocab=vocab, pad=pad, f32=f32, inv_temp=inv_temp, ignored=ignored, **kw)


def _head(rows, vocab, d, f32=False, inv_temp=1.0, ignored=0.0):
    return dict(op="head", rows=rows, vocab=vocab, d=d, f32=f32, inv_temp=inv_temp, ignored=ignored)


def _policy(seqs, length, ref=True, entropy=True, seq_mean=False, token_adv=False, norm=0.0):
    return dict(op="policy", seqs=seqs, length=length, ref=ref, entropy=entropy, seq_mean=seq_mean,
                token_adv=token_adv, norm=norm)


def _pref(pairs, length, ref=True, kind="sigmoid", smoothing=0.0, margin=0.0, normalize=False):
    return dict(op="preference", pairs=pairs, length=length, ref=ref, kind=kind, smoothing=smoothing,
                margin=margin, normalize=normalize)


def listed():
    return [
        # the log-probability of one sampled token at a large vocabulary: latency
        dict(_rows("logprob", 1, 128256, f32=False, inv_temp=1.25), name="logprob-one-row"),
        # a microbatch of a last stage (8 x 1024 tokens, fp32 logits), prompt tokens ignored
        dict(_rows("logprob", 8192, 49152, ignored=0.25), name="logprob-last-stage"),
        # the gradient where neither the token count nor the vocabulary is a multiple of anything,
        # with an entropy term, to bf16
        dict(_rows("logprob_grad", 999, 32001, ignored=0.1, out_f32=False, entropy=True, inv_temp=1.25),
             name="grad-odd"),
        # bf16 logits of a large vocabulary, their gradient in bf16
        dict(_rows("logprob_grad", 4096, 128256, f32=False, ignored=0.25, out_f32=False, entropy=False),
             name="grad-large-vocab"),
        # one new token's hidden state through the head: the head's matrix is read once
        dict(_head(1, 128256, 4096), name="head-one-token"),
        # an fp32 stage of an odd token count
        dict(_head(333, 32001, 512, f32=True, ignored=0.1), name="head-odd-f32"),
        # scoring a microbatch with a frozen reference policy, no gradient
        dict(_head(8192, 49152, 2048, ignored=0.0), name="head-score"),
        # a handful of short answers: launches
        dict(_policy(4, 64, entropy=False), name="policy-few"),
        # one update over 512 answers of up to 4096 tokens
        dict(_policy(512, 4096, token_adv=True), name="policy-many"),
        # odd lengths, every answer weighing the same
        dict(_policy(37, 1111, seq_mean=True), name="policy-odd"),
        # a microbatch of two short pairs
        dict(_pref(2, 100), name="preference-few"),
        # 256 pairs of up to 4096 tokens, lengths normalised, label smoothing
        dict(_pref(256, 4096, smoothing=0.1, normalize=True), name="preference-many"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprob", "logprob_grad", "head", "policy", "preference"])
    temp, ignored = rng.choice([1.0, 1.25, 0.625, 2.0]), rng.choice([0.0, 0.1, 0.5])
    if op in ("logprob", "logprob_grad"):
        vocab = _log(rng, 32, 131072)
        rows = _log(rng, 1, min(16384, 4.0e8 / vocab))
        c = _rows(op, rows, vocab, rng.choice([0, 0, 1, 7, 64]), rng.random() < 0.5, temp, ignored)
        if op == "logprob_grad":
            c.update(out_f32=rng.random() < 0.5, entropy=rng.random() < 0.5)
        return c
    if op == "head":
        vocab, d, f32 = _log(rng, 32, 131072), 8 * _log(rng, 8, 512), rng.random() < 0.25
        rows = _log(rng, 1, min(8192, (1.0e11 if f32 else 8.0e11) / (vocab * d)))
        return _head(rows, vocab, d, f32, temp, ignored)
    if op == "policy":
        length = _log(rng, 1, 16384)
        return _policy(_log(rng, 1, max(1, min(2048, 2.0e6 / length))), length, rng.random() < 0.7,
                       rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.5,
                       rng.choice([0.0, 0.0, 4096.0]))
    length, kind = _log(rng, 1, 16384), rng.choice(["sigmoid", "sigmoid", "hinge", "square"])
    return _pref(_log(rng, 1, max(1, min(1024, 1.0e6 / length))), length, rng.random() < 0.7, kind,
                 rng.choice([0.0, 0.1]) if kind == "sigmoid" else 0.0, rng.choice([0.0, 0.5]), rng.random() < 0.5)


# ------------------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _targets(case, g):
    """One target per row; a fixed share of the rows, anywhere, has none (-1)."""
    n, k = case["rows"], int(case["rows"] * case["ignored"])
    t = torch.randint(0, case["vocab"], (n,), generator=g, device=DEV, dtype=torch.int32)
    t[torch.randperm(n, generator=g, device=DEV)[:k]] = -1
    return t


def _row_outputs(n):
    f = dict(dtype=torch.float32, device=DEV)
    return dict(logp=torch.empty(n, **f), entropy=torch.empty(n, **f), stats=torch.empty(n, 2, **f))


def _response_mask(n, length, g):
    """Answers of random lengths after prompts of random lengths; one in sixteen has no token."""
    start = (torch.rand(n, 1, generator=g, device=DEV) * 0.4 * length).long()
    stop = start + 1 + (torch.rand(n, 1, generator=g, device=DEV) * (length - start)).long()
    t = torch.arange(length, device=DEV)[None, :]
    empty = torch.rand(n, 1, generator=g, device=DEV) < 1 / 16
    if n <= 2:
        empty[:] = False
    return ((t >= start) & (t < stop) & ~empty).to(torch.uint8)


def _logps(shape, g):
    """Log-probabilities of sampled tokens: most near 0, a long tail."""
    u = torch.rand(shape, generator=g, device=DEV)
    return -(-torch.log1p(-u * 0.9999)) ** 2


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    op = case["op"]
    if op in ("logprob", "logprob_grad"):
        n, v = case["rows"], case["vocab"]
        dt = torch.float32 if case["f32"] else torch.bfloat16
        t = _targets(case, g)
        x = torch.empty(n, v + case["pad"], dtype=dt, device=DEV).normal_(0.0, 2.0, generator=g)
        peak = torch.rand(n, generator=g, device=DEV) * 14.0  # sampled tokens are likely ones
        x[torch.arange(n, device=DEV), t.clamp(min=0).long()] += peak.to(dt)
        x = x[:, :v]
        s.update(logits=x, targets=t)
        if op == "logprob":
            s["out"] = _row_outputs(n)
        else:
            # what the forward left, and a gradient as a loss over the batch gives it
            m = x.float().amax(1)
            z = (x.float() - m[:, None]) * case["inv_temp"]
            logs = torch.log(torch.exp(z).sum(1, dtype=torch.float64))
            q = z.double() - logs[:, None]
            ent = -(q.exp() * q).sum(1)
            on = t >= 0
            s["stats"] = torch.where(on[:, None], torch.stack([m, logs.float()], 1), 0.0)
            s["entropy"] = torch.where(on, ent.float(), 0.0)
            s["logp"] = torch.where(on, q.gather(1, t.clamp(min=0).long()[:, None])[:, 0].float(), 0.0)
            s["dlogp"] = torch.randn(n, generator=g, device=DEV) / n
            s["dentropy"] = torch.full((n,), -0.01 / n, device=DEV) if case["entropy"] else None
            s["dlogits"] = torch.empty(n, v, dtype=torch.float32 if case["out_f32"] else torch.bfloat16, device=DEV)
    elif op == "head":
        n, v, d = case["rows"], case["vocab"], case["d"]
        dt = torch.float32 if case["f32"] else torch.bfloat16
        s["targets"] = _targets(case, g)
        s["x"] = torch.empty(n, d, dtype=dt, device=DEV).normal_(0.0, 1.0, generator=g)
        s["weight"] = torch.empty(v, d, dtype=dt, device=DEV).normal_(0.0, 2.0 / math.sqrt(d), generator=g)
        s["out"] = _row_outputs(n)
    elif op == "policy":
        b, n = case["seqs"], case["length"]
        logp = _logps((b, n), g)
        s.update(logp=logp, mask=_response_mask(b, n, g),
                 old=logp + 0.15 * torch.randn(b, n, generator=g, device=DEV),
                 ref=logp + 0.3 * torch.randn(b, n, generator=g, device=DEV) if case["ref"] else None,
                 entropy=-0.5 * logp if case["entropy"] else None,
                 adv=torch.randn((b, n) if case["token_adv"] else (b,), generator=g, device=DEV),
                 clip_low=_f32(0.2), clip_high=_f32(0.28), kl=_f32(0.05) if case["ref"] else 0.0,
                 ent=_f32(0.01) if case["entropy"] else 0.0)
        s["out"] = dict(loss=torch.empty(1, device=DEV), dlogp=torch.empty(b, n, device=DEV),
                        dentropy=torch.empty(b, n, device=DEV) if case["entropy"] else None,
                        metrics=torch.empty(6, device=DEV),
                        counts=torch.empty(2, dtype=torch.int64, device=DEV))
    else:
        p, n = case["pairs"], case["length"]
        logp = _logps((2 * p, n), g)
        # a policy some steps from its reference: a common shift per answer and noise per token
        shift = torch.randn(2 * p, 1, generator=g, device=DEV) * (2.0 / n)
        s.update(logp=logp, mask=_response_mask(2 * p, n, g),
                 ref=logp - shift + 0.02 * torch.randn(2 * p, n, generator=g, device=DEV) if case["ref"] else None,
                 beta=_f32(2.0 if case["normalize"] else 0.1), smoothing=_f32(case["smoothing"]),
                 margin=_f32(case["margin"]))
        s["out"] = dict(loss=torch.empty(1, device=DEV), dlogp=torch.empty(2 * p, n, device=DEV),
                        pair_loss=torch.empty(p, device=DEV), rewards=torch.empty(2 * p, device=DEV),
                        metrics=torch.empty(4, device=DEV),
                        counts=torch.empty(1, dtype=torch.int64, device=DEV))
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_logprob(x, t, inv_temp):
    on = t >= 0
    z = x.float()
    m = z.amax(1)
    z = (z - m[:, None]) * inv_temp
    e = torch.exp(z)
    total = e.sum(1)
    logs = torch.log(total)
    logp = z.gather(1, t.clamp(min=0).long()[:, None])[:, 0] - logs
    ent = logs - (e * z).sum(1) / total
    return dict(logp=torch.where(on, logp, 0.0), entropy=torch.where(on, ent, 0.0),
                stats=torch.where(on[:, None], torch.stack([m, logs], 1), 0.0))


def _plain_grad(s):
    c, t = s["case"], s["targets"]
    st = s["stats"]
    on = t >= 0
    q = (s["logits"].float() - st[:, :1]) * c["inv_temp"] - st[:, 1:]
    p = torch.exp(q)
    d = -p * s["dlogp"][:, None]
    d[torch.arange(c["rows"], device=DEV), t.clamp(min=0).long()] += s["dlogp"]
    if s["dentropy"] is not None:
        d = d - s["dentropy"][:, None] * p * (q + s["entropy"][:, None])
    d = torch.where(on[:, None], d * c["inv_temp"], 0.0)
    return dict(dlogits=d.to(s["dlogits"].dtype))


def _plain_policy(s):
    c = s["case"]
    on = s["mask"] != 0
    n_b = on.sum(1)
    tokens, seqs = on.sum(), (n_b > 0).sum()
    if c["seq_mean"]:
        den = c["norm"] if c["norm"] > 0 else seqs.clamp(min=1).double()
        w = (1.0 / (den * n_b.clamp(min=1).double()))[:, None].float()
    else:
        den = c["norm"] if c["norm"] > 0 else tokens.clamp(min=1).double()
        w = (torch.ones(1, 1, dtype=torch.float64, device=DEV) / den).float()
    adv = s["adv"] if c["token_adv"] else s["adv"][:, None]
    # the differences in 64 bits: which side of the clip a token is on, and the KL terms near 0
    x = s["logp"].double() - s["old"].double()
    cut = ((x > math.log1p(s["clip_high"])) & (adv > 0)) | ((x < math.log1p(-s["clip_low"])) & (adv < 0))
    r = torch.exp(x.float())
    surr = -torch.where(cut, r.clamp(1.0 - s["clip_low"], 1.0 + s["clip_high"]), r) * adv
    g = torch.where(cut, 0.0, -r * adv)
    kl_old = (torch.expm1(x) - x).float()
    kl = torch.zeros((), device=DEV)
    if s["ref"] is not None:
        d = s["ref"].double() - s["logp"].double()
        kl = (torch.expm1(d) - d).float()
        g = g - s["kl"] * torch.expm1(d.float())
    ent = s["entropy"] if s["entropy"] is not None else torch.zeros((), device=DEV)
    total = lambda v: (w * torch.where(on, v, 0.0)).sum(dtype=torch.float64)  # noqa: E731
    surr, kl, ent = total(surr), total(kl), total(ent)
    loss = surr + s["kl"] * kl - s["ent"] * ent
    met = torch.stack([surr, kl, ent, total(cut.float()), total(kl_old), total(r)])
    out = dict(loss=loss.float().reshape(1), dlogp=torch.where(on, w * g, 0.0), metrics=met.float(),
               counts=torch.stack([tokens, seqs]))
    if s["entropy"] is not None:
        out["dentropy"] = torch.where(on, -s["ent"] * w, 0.0)
    return out


def _plain_preference(s):
    c = s["case"]
    on = s["mask"] != 0
    n = on.sum(1)
    v = s["logp"].double() if s["ref"] is None else s["logp"].double() - s["ref"].double()
    size = n.clamp(min=1).double() if c["normalize"] else torch.ones(1, dtype=torch.float64, device=DEV)
    score = torch.where(on, v, 0.0).sum(1) / size
    p = c["pairs"]
    live = (n[:p] > 0) & (n[p:] > 0)
    count = live.sum().clamp(min=1).double()
    delta = score[:p] - score[p:]
    h = s["beta"] * delta - s["margin"]
    if c["kind"] == "sigmoid":
        soft = lambda u: torch.log1p(torch.exp(-u.abs())) + u.clamp(min=0.0)  # noqa: E731
        loss = (1.0 - s["smoothing"]) * soft(-h) + s["smoothing"] * soft(h)
        dh = s["smoothing"] - 1.0 / (1.0 + torch.exp(h))
    elif c["kind"] == "hinge":
        loss = (1.0 - h).clamp(min=0.0)
        dh = -(h < 1.0).double()
    else:
        loss = ((h - 0.5) / s["beta"]) ** 2
        dh = 2.0 * (h - 0.5) / s["beta"] ** 2
    pick = lambda u: torch.where(live, u, 0.0)  # noqa: E731
    loss, dh = pick(loss), pick(dh) * s["beta"] / count
    two = torch.cat([live, live])
    rewards = torch.where(two, s["beta"] * score, 0.0)
    met = torch.stack([pick((delta > 0).double()).sum() / count, rewards[:p].sum() / count,
                       rewards[p:].sum() / count, pick(h).sum() / count])
    dlogp = torch.where(on, (torch.cat([dh, -dh]) / size)[:, None], 0.0)
    return dict(loss=(loss.sum() / count).float().reshape(1), dlogp=dlogp.float(), pair_loss=loss.float(),
                rewards=rewards.float(), metrics=met.float(), counts=live.sum().reshape(1))


# ------------------------------------------------------------------------------------------ run
def run(state):
    s, c = state, state["case"]
    if not own:
        if c["op"] == "logprob":
            return _plain_logprob(s["logits"], s["targets"], c["inv_temp"])
        if c["op"] == "logprob_grad":
            return _plain_grad(s)
        if c["op"] == "head":
            return _plain_logprob(s["x"].float() @ s["weight"].float().t(), s["targets"], c["inv_temp"])
        if c["op"] == "policy":
            return _plain_policy(s)
        return _plain_preference(s)
    from paper_2606_30634_amd import losses
    if c["op"] == "logprob":
        out = losses.LogProb(**s["out"])
        losses.token_logprob(s["logits"], s["targets"], inv_temperature=c["inv_temp"], out=out)
        return s["out"]
    if c["op"] == "logprob_grad":
        fwd = losses.LogProb(s["logp"], s["entropy"], s["stats"])
        losses.token_logprob_backward(s["logits"], s["targets"], fwd, s["dlogp"], s["dentropy"],
                                      inv_temperature=c["inv_temp"], out=s["dlogits"])
        return dict(dlogits=s["dlogits"])
    if c["op"] == "head":
        out = losses.LogProb(**s["out"])
        losses.head_logprob(s["x"], s["weight"], s["targets"], inv_temperature=c["inv_temp"], out=out)
        return s["out"]
    if c["op"] == "policy":
        out = losses.PolicyLoss(**s["out"])
        losses.policy_loss(s["logp"], s["old"], s["adv"], s["mask"], ref_logp=s["ref"], entropy=s["entropy"],
                           clip_low=s["clip_low"], clip_high=s["clip_high"], kl_coef=s["kl"],
                           entropy_coef=s["ent"], reduction="sequence" if c["seq_mean"] else "token",
                           norm=c["norm"], out=out)
        return s["out"]
    out = losses.PreferenceLoss(**s["out"])
    losses.preference_loss(s["logp"], s["mask"], ref_logp=s["ref"], kind=c["kind"], beta=s["beta"],
                           label_smoothing=s["smoothing"], margin=s["margin"], length_normalize=c["normalize"],
                           out=out)
    return s["out"]


# ------------------------------------------------------------------------------------------ work
def work(case):
    c = case
    e = 4 if c.get("f32", True) else 2
    if c["op"] in ("logprob", "logprob_grad"):
        read = (c["rows"] - int(c["rows"] * c["ignored"])) * c["vocab"]
        if c["op"] == "logprob":
            return dict(bytes=read * e + c["rows"] * 20, flops=5 * read)
        write = c["rows"] * c["vocab"] * (4 if c["out_f32"] else 2)
        return dict(bytes=read * e + write + c["rows"] * 24, flops=6 * read)
    if c["op"] == "head":
        live = c["rows"] - int(c["rows"] * c["ignored"])
        return dict(bytes=(live + c["vocab"]) * c["d"] * e + c["rows"] * 20, flops=2 * live * c["vocab"] * c["d"])
    # every mask byte and gradient, the inputs of the tokens that count (0.375 of them on average)
    if c["op"] == "policy":
        n = c["seqs"] * c["length"]
        live = int(0.375 * n) + 1
        per = 8 + 4 * c["ref"] + 4 * c["entropy"] + 4 * c["token_adv"]
        return dict(bytes=live * per + n * (5 + 4 * c["entropy"]) + 4 * c["seqs"] + 44, flops=20 * live)
    n = 2 * c["pairs"] * c["length"]
    live = int(0.375 * n) + 1
    return dict(bytes=live * (4 + 4 * c["ref"]) + 5 * n + 12 * c["pairs"] + 24, flops=4 * live)


# ------------------------------------------------------------------------------------------ exact
def _exact_rows(x, t, inv_temp):
    """Log-probabilities, entropies and statistics of rows of 64-bit logits."""
    on = t >= 0
    z = x * inv_temp
    m = z.amax(1)
    lse = torch.logsumexp(z, 1)
    q = z - lse[:, None]
    ent = -(q.exp() * q).sum(1)
    logp = q[torch.arange(z.shape[0], device=DEV), t.clamp(min=0).long()]
    keep = lambda v: torch.where(on, v, torch.zeros_like(v))  # noqa: E731
    return dict(logp=keep(logp), entropy=keep(ent), stats=torch.stack([keep(x.amax(1)), keep(lse - m)], 1))


def exact(case, seed):
    s = prepare(case, seed)
    op, c = case["op"], case
    if op == "logprob":
        return _exact_rows(s["logits"].double(), s["targets"], c["inv_temp"])
    if op == "head":
        x = s["x"].double() @ s["weight"].double().t()
        return _exact_rows(x, s["targets"], c["inv_temp"])
    if op == "logprob_grad":
        x = s["logits"].double().requires_grad_(True)
        q = torch.log_softmax(x * c["inv_temp"], 1)
        on = (s["targets"] >= 0).double()
        picked = q.gather(1, s["targets"].clamp(min=0).long()[:, None])[:, 0]
        obj = (picked * on * s["dlogp"].double()).sum()
        if s["dentropy"] is not None:
            obj = obj + (-(q.exp() * q).sum(1) * on * s["dentropy"].double()).sum()
        obj.backward()
        return dict(dlogits=x.grad)
    on = s["mask"] != 0
    count = on.double().sum(1)
    if op == "policy":
        lp = s["logp"].double().requires_grad_(True)
        ent = s["entropy"].double().requires_grad_(True) if s["entropy"] is not None else None
        inside = on.nonzero(as_tuple=True)  # only the tokens that count
        adv = s["adv"].double() if c["token_adv"] else s["adv"].double()[:, None].expand_as(lp)
        if c["seq_mean"]:
            per = 1.0 / count[inside[0]]
            per = per / (c["norm"] if c["norm"] > 0 else max(1, int((count > 0).sum())))
        else:
            per = torch.ones_like(count[inside[0]]) / (c["norm"] if c["norm"] > 0 else max(1, int(on.sum())))
        x = lp[inside] - s["old"].double()[inside]
        a = adv[inside]
        bound = torch.where(a >= 0, torch.clamp(x.exp(), max=1.0 + s["clip_high"]),
                            torch.clamp(x.exp(), min=1.0 - s["clip_low"]))
        surr = -(per * bound * a).sum()
        zero = torch.zeros((), dtype=torch.float64, device=DEV)
        kl = ent_s = zero
        if s["ref"] is not None:
            d = s["ref"].double()[inside] - lp[inside]
            kl = (per * (torch.expm1(d) - d)).sum()
        if ent is not None:
            ent_s = (per * ent[inside]).sum()
        loss = surr + s["kl"] * kl - s["ent"] * ent_s
        loss.backward()
        with torch.no_grad():
            cut = ((a > 0) & (x > math.log1p(s["clip_high"]))) | ((a < 0) & (x < math.log1p(-s["clip_low"])))
            met = torch.stack([surr, kl, ent_s, (per * cut).sum(), (per * (torch.expm1(x) - x)).sum(),
                               (per * x.exp()).sum()])
            counts = torch.stack([on.sum(), (count > 0).sum()])
        out = dict(loss=loss.detach().reshape(1), dlogp=lp.grad, metrics=met, counts=counts)
        if ent is not None:
            out["dentropy"] = ent.grad
        return out
    lp = s["logp"].double().requires_grad_(True)
    p = c["pairs"]
    v = lp if s["ref"] is None else lp - s["ref"].double()
    score = (v * on).sum(1)
    if c["normalize"]:
        score = score / count.clamp(min=1)
    live = ((count[:p] > 0) & (count[p:] > 0)).nonzero()[:, 0]
    k = max(1, live.numel())
    delta = score[:p][live] - score[p:][live]
    h = s["beta"] * delta - s["margin"]
    if c["kind"] == "sigmoid":
        each = (-(1.0 - s["smoothing"]) * torch.nn.functional.logsigmoid(h)
                - s["smoothing"] * torch.nn.functional.logsigmoid(-h))
    elif c["kind"] == "hinge":
        each = torch.relu(1.0 - h)
    else:
        each = (delta - s["margin"] / s["beta"] - 0.5 / s["beta"]) ** 2
    loss = each.sum() / k
    loss.backward()
    with torch.no_grad():
        pair = torch.zeros(p, dtype=torch.float64, device=DEV).index_copy(0, live, each.detach())
        rewards = torch.zeros(2 * p, dtype=torch.float64, device=DEV)
        rewards[live] = s["beta"] * score[live].detach()
        rewards[live + p] = s["beta"] * score[live + p].detach()
        met = torch.stack([(delta > 0).double().sum() / k, rewards[:p].sum() / k, rewards[p:].sum() / k,
                           h.sum() / k])
        counts = torch.tensor([live.numel()], device=DEV)
    return dict(loss=loss.detach().reshape(1), dlogp=lp.grad, pair_loss=pair, rewards=rewards, metrics=met,
                counts=counts)
