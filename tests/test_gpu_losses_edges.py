"""Log-probability and loss operators at edges of their own: inputs taken in chunks, workspaces of exactly the size
asked for, values at the ends of the types.  Against the oracle in float64; bounds count roundings, u = 2^-24, as the
operators' other tests do."""
import numpy as np
import pytest

from gpu_common import log
from oracle import losses as L
from test_gpu_losses import U, _err, _f32, _head_tol, _i32, _matrix, _np

pytestmark = pytest.mark.gpu


def _guarded(need, guard=65536):
    """A uint8 workspace of `need` bytes with a pattern behind it, and the check that the pattern is whole."""
    import torch
    buf = torch.full((need + guard,), 0xA5, dtype=torch.uint8, device="cuda:0")
    return buf[:need], lambda: bool((buf[need:] == 0xA5).all())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,v,d", [(712, 16384, 33), (600, 20000, 33), (129, 128256, 33), (99, 128256, 5), (1300, 8193, 1)])
def test_head_of_unaligned_rows_in_chunks(n, v, d, bf16):
    """Rows that are not whole 16 bytes go through fp32 logits, 32 MiB of them at a time: several chunks, the last of
    them smaller and split further than the others.  Nothing is written behind the workspace."""
    from paper_2606_30634_amd import binding as B
    from paper_2606_30634_amd import losses
    r = np.random.default_rng(n + v)
    mx, xv = _matrix(r.normal(size=(n, d)), bf16, pad=2)
    mw, wv = _matrix(r.normal(size=(v, d)) * (2 / np.sqrt(d)), bf16, lead=1)
    t = r.integers(0, v, size=n)
    t[n // 3], t[n - 2] = -1, v
    rows = np.unique(np.r_[0:n:37, n // 3, n // 2, n - 34:n])  # the oracle's share of them
    log(f"rows {n} vocab {v} d {d} bf16 {bf16}")
    need = B.head_logprob_workspace_bytes(n, v, d, bf16)
    ws, whole = _guarded(need)
    got = losses.head_logprob(mx, mw, _i32(t), inv_temperature=1.5, workspace=ws)
    assert whole()
    ref = L.token_logprob(xv[rows] @ wv.T, t[rows], 1.5)
    e = _head_tol(d, xv[rows], wv, 1.5)
    lp, ent, st = (_np(a)[rows] for a in got)
    assert (np.abs(lp - ref[0]) <= 2 * e + _err(v, ref[0])).all()
    assert (np.abs(st[:, 0] - ref[2][:, 0]) <= e / 1.5).all()
    assert (np.abs(st[:, 1] - ref[2][:, 1]) <= 2 * e + _err(v, 0.0)).all()
    assert (np.abs(ent - ref[1]) <= (2 * e + 2 * _err(v, 0.0)) * 2 * (np.abs(ref[2][:, 1]) + 1 + np.log(v))).all()
    gone = (t < 0) | (t >= v)
    assert gone.sum() == 2 and not _np(got.logp)[gone].any() and _np(got.logp)[~gone].all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,v,d", [(1, 300, 64), (24, 30000, 64), (45, 10902, 2144), (300, 777, 1000), (333, 32001, 512),
                                   (16400, 264, 64), (700, 9001, 2996)])
def test_head_workspace_is_enough(n, v, d, bf16):
    """Every way the fused product lays out its workspace: row tiles, packed rows, more rows than one product takes."""
    import torch
    from paper_2606_30634_amd import binding as B
    from paper_2606_30634_amd import losses
    g = torch.Generator(device="cuda:0").manual_seed(n)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = torch.randn(n, d, generator=g, device="cuda:0").to(dt)
    w = (torch.randn(v, d, generator=g, device="cuda:0") / d ** 0.5).to(dt)
    t = torch.randint(-v // 4, v, (n,), generator=g, device="cuda:0", dtype=torch.int32)
    log(f"rows {n} vocab {v} d {d} bf16 {bf16}")
    ws, whole = _guarded(B.head_logprob_workspace_bytes(n, v, d, bf16))
    got = losses.head_logprob(x, w, t, workspace=ws)
    assert whole()
    other = losses.head_logprob(x, w, t)
    assert all(torch.equal(a, b) for a, b in zip(got, other))


def test_other_workspaces_are_enough():
    """Rows of logits in parts, and the losses above and below the sizes that one block takes."""
    import torch
    from paper_2606_30634_amd import binding as B
    from paper_2606_30634_amd import losses
    for n, v in ((1, 16384), (5, 40001), (34, 128256), (256, 16390), (513, 20000)):
        log(f"rows {n} vocab {v}")
        x = torch.randn(n, v, device="cuda:0")
        t = torch.randint(-2, v, (n,), device="cuda:0", dtype=torch.int32)
        ws, whole = _guarded(B.token_logprob_workspace_bytes(n, v))
        losses.token_logprob(x, t, workspace=ws)
        assert whole()
    for b, s in ((1, 1), (8, 1024), (9, 1024), (1026, 3), (2, 40001), (600, 2048), (70000, 2)):
        log(f"sequences {b} length {s}")
        lp = -torch.rand(b, s, device="cuda:0")
        on = torch.rand(b, s, device="cuda:0") < 0.7
        ws, whole = _guarded(B.policy_loss_workspace_bytes(b, s))
        losses.policy_loss(lp, lp + 0.1, lp[:, 0].contiguous(), on, workspace=ws)
        assert whole()
        if b % 2 == 0:
            ws, whole = _guarded(B.preference_loss_workspace_bytes(b // 2, s))
            losses.preference_loss(lp, on, workspace=ws)
            assert whole()


# ------------------------------------------------------------------ from hidden states
def _one_hot(n, d, bf16):
    """Hidden states that pick a column of the head's matrix each, so that a product's logits are its elements."""
    import torch
    x = torch.zeros(n, d, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    x[torch.arange(n), torch.arange(n) % d] = 1
    return x


TILES = [(True, 64, 128, 64), (True, 130, 257, 40), (True, 1152, 4096, 1024), (True, 2944, 1024, 64), (True, 2000, 6001, 520),
         (True, 32, 25856, 64), (True, 7, 26001, 72), (False, 64, 128, 64), (False, 130, 257, 40), (False, 1024, 4096, 256),
         (False, 2000, 4001, 772), (False, 32, 1280, 64), (False, 5, 1001, 68), (True, 5, 40, 64), (False, 3, 700, 33)]


@pytest.mark.parametrize("bf16,n,v,d", TILES)
def test_head_target_of_probability_near_one(bf16, n, v, d):
    """log p of a target that has nearly all of its row is -log(1 + s), s the others' sum of some 2^-20, to s's own
    relative accuracy.  The logits are exact.  A term of s: its exponent t < 2^5 rounded, 2^5 log 2 u, and exp2's 2 u; the
    sum: at most 32 additions of a lane and 4 of lanes, then merges of 3 roundings, at most v / 512 + 16 of them (panels of
    32 columns or more, 16 threads or more on a row, 4 steps in a wave, 3 across, and those of rows in parts); the logarithm
    and the last products 8 u."""
    import torch
    from paper_2606_30634_amd import losses
    r = np.random.default_rng(n + v + d)
    w = np.minimum(r.normal(size=(v, d)), 2.0)
    tk = r.integers(0, v, size=d)
    w[tk, np.arange(d)] = 16.0 + np.floor(np.log(v))
    mw, wv = _matrix(w, bf16)
    k = np.arange(n) % d
    got = losses.head_logprob(_one_hot(n, d, bf16), mw, _i32(tk[k]))
    z = wv - wv[tk, np.arange(d)][None]
    e = np.exp(z)
    e[tk, np.arange(d)] = 0.0
    s = e.sum(0)
    assert (s < 2.0 ** -10).all()
    tol = (22 + 2 + 36 + 3 * (v / 512 + 16) + 8) * U
    for name, g, want, rel in (("logp", got.logp, -np.log1p(s), tol),
                               ("entropy", got.entropy, np.log1p(s) - (e * z).sum(0) / (1 + s), 2 * tol)):
        d_ = np.abs(_np(g) - want[k]) / np.abs(want[k])
        assert d_.max() <= rel, (name, d_.max(), rel)
    assert torch.equal(got.stats[:, 0].double().cpu(), torch.from_numpy(wv[tk, np.arange(d)][k]))


@pytest.mark.parametrize("bf16,n,v,d", TILES)
def test_head_of_several_largest_logits(bf16, n, v, d):
    """Rows whose largest logit stands in 1, 2, 3 or 5 places, in one panel or in several: exact counts, log p = -log 5
    and the like, beside logits so low that they add nothing."""
    from paper_2606_30634_amd import losses
    r = np.random.default_rng(n)
    w = np.full((v, d), -200.0)
    c = np.array([1, 2, 3, 5])[np.arange(d) % 4]
    tk = np.zeros(d, np.int64)
    for j in range(d):
        first = int(r.integers(0, v - 5))
        at = first + np.arange(c[j]) if j % 8 < 4 else r.choice(v, size=c[j], replace=False)
        w[at, j], tk[j] = 7.0, at[-1]
    mw, _ = _matrix(w, bf16)
    k = np.arange(n) % d
    got = losses.head_logprob(_one_hot(n, d, bf16), mw, _i32(tk[k]))
    want = np.log(c[k].astype(float))
    assert (np.abs(_np(got.logp) + want) <= 4 * U * want).all() and (np.abs(_np(got.entropy) - want) <= 4 * U * want).all()


@pytest.mark.parametrize("bf16,n,v,d", TILES)
def test_head_of_masks_and_nonfinite_values(bf16, n, v, d):
    """-inf, the type's lowest value, +inf and NaN among the logits of a head, at both ends of the vocabulary and inside it:
    as for rows of logits."""
    import torch
    from paper_2606_30634_amd import losses
    r = np.random.default_rng(v)
    lowest = float(torch.finfo(torch.bfloat16 if bf16 else torch.float32).min)
    w = np.minimum(r.normal(size=(v, d)) * 2, 6.0)
    kinds = np.arange(d) % 6
    tk = r.integers(0, v, size=d)
    w[:, kinds == 1] = lowest                                  # uniform
    for j in np.nonzero(kinds == 2)[0]:                        # one token left
        w[:, j] = lowest
        w[tk[j], j] = 3.0
    w[::2, kinds == 3] = lowest                                # every other one masked
    w[-1, kinds == 4] = lowest
    w[:, kinds == 5] += 3e4                                    # large logits
    mw, wv = _matrix(w, bf16)
    x = _one_hot(n, d, bf16)
    k = np.arange(n) % d
    ref = L.token_logprob(wv.T.copy(), tk, 1.0)

    def check(got, rows):
        for g, want, tol in zip(got, ref, (_err(v, ref[0]), 2 * _err(v, 0.0) * (np.abs(ref[2][:, 1]) + 1 + np.log(v)),
                                           np.full((d, 1), _err(v, 0.0)))):
            g, want, tol = _np(g)[rows], want[k][rows], np.asarray(tol)[k][rows]
            assert (np.abs(g - want) <= tol).all(), np.abs(g - want).max()
        assert (_np(got.stats)[rows, 0] == ref[2][k][rows, 0]).all()
    got = losses.head_logprob(x, mw, _i32(tk[k]))
    check(got, np.ones(n, bool))
    # a hidden state with a NaN or an infinity makes its own row NaN and no other
    x[0, 0] = float("nan")
    x[n - 1, d - 1] = float("inf")
    got = losses.head_logprob(x, mw, _i32(tk[k]))
    for row in (0, n - 1):
        with np.errstate(invalid="ignore"):
            z = _np(x[row]) @ wv.T
        if (np.isnan(z) | (z == np.inf)).any():
            assert np.isnan(_np(got.logp)[row]) and np.isnan(_np(got.entropy)[row])
        else:  # the infinity met only negative elements
            assert (z == -np.inf).all() and _np(got.logp)[row] == -np.inf and _np(got.entropy)[row] == 0
    check(got, np.arange(n) % (n - 1) != 0)
    # rows of the head's matrix that are -inf: tokens that cannot occur; nothing else: no distribution
    x = torch.ones_like(x)
    wi, t = wv.copy(), tk[k]
    wi[: v // 2] = -np.inf
    wi[-1] = -np.inf
    t = np.where(t < v // 2, 0, np.minimum(t, v - 2))
    mw, wiv = _matrix(wi / 64, bf16)
    got = losses.head_logprob(x, mw, _i32(t))
    z = wiv.sum(1)
    z[z < np.finfo(np.float32).min] = -np.inf  # a product past fp32, of a wide head's masks
    with np.errstate(invalid="ignore"):
        one = L.token_logprob(np.repeat(z[None], n, 0), t, 1.0)
    assert (_np(got.logp)[one[0] == -np.inf] == -np.inf).all() and (one[0][t == 0] == -np.inf).all()
    e = 2 * U * (d + 2) * float(np.abs(wiv[np.isfinite(wiv).all(1)]).sum(1).max())
    fin = np.isfinite(one[0])
    assert (np.abs(_np(got.logp)[fin] - one[0][fin]) <= e + _err(v, one[0][fin])).all()
    assert (np.abs(_np(got.entropy) - one[1]) <= (e + 2 * _err(v, 0.0)) * 2 * (1 + np.log(v) + one[2][:, 1])).all()
    got = losses.head_logprob(x, torch.full_like(mw, -torch.inf), _i32(t))
    assert bool((got.logp == -torch.inf).all()) and not bool(got.entropy.any())
    assert bool((got.stats[:, 0] == -torch.inf).all()) and not bool(got.stats[:, 1].any())


# ------------------------------------------------------------------ the target's own term
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("path", ["rows", "parts", "head"])
def test_log_probability_of_a_far_target(path, bf16):
    """s (x_t - m) beside a log-sum that is nearly nothing: with m = 0 and s = 1 the difference and the product are exact
    and log p is rounded once, u of it; with another s twice.  The log-sum's own 8 u come on top."""
    import torch
    from paper_2606_30634_amd import losses
    r = np.random.default_rng(3)
    n, v = 64, 40000 if path == "parts" else 96
    x = np.full((n, v), -150.0)
    x[np.arange(n), r.integers(0, v // 2, size=n)] = 0.0
    t = v // 2 + r.integers(0, v // 2, size=n)
    x[np.arange(n), t] = -r.uniform(9, 90, size=n)
    for s, roundings in ((1.0, 1), (1.3, 2)):
        if path == "head":  # a row of the identity per logit row
            mx, xv = _matrix(x.T.copy(), bf16)
            got = losses.head_logprob(_one_hot(n, n, bf16), mx, _i32(t), inv_temperature=s)
            xv = xv.T
        else:
            mx, xv = _matrix(x, bf16)
            got = losses.token_logprob(mx, _i32(t), inv_temperature=s)
        sf = float(np.float32(s))
        ls = np.log1p(np.exp(sf * xv[np.arange(n), t]))
        want = sf * xv[np.arange(n), t] - ls
        d = np.abs(_np(got.logp) - want)
        assert (d <= roundings * U * np.abs(want) * (1 + 2.0 ** -20) + 8 * U * ls).all(), (s, (d / np.abs(want)).max() / U)


# ------------------------------------------------------------------ masked logits under a large upstream gradient
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("v", [6, 700, 40001])
def test_entropy_gradient_of_masked_logits_at_large_scales(v, bf16):
    """-inf logits, and ones s takes past the type's range, have p = 0 and so no entropy gradient, however large s times
    dentropy is."""
    import torch
    from paper_2606_30634_amd import losses
    r = np.random.default_rng(v)
    n = 5
    x = r.normal(size=(n, v))
    x[:, ::2] = -np.inf
    x[:, 1], x[:, 5] = 4.0, 4.0  # two tokens share the row where s is large
    t = np.array([1, 1, 0, 3, 5])  # the third cannot occur
    x[3, 3] = 4.0
    mx, xv = _matrix(x, bf16)
    g, gv = _f32(r.normal(size=n))
    for s, dent in ((2.0 ** 40, 1e-2), (2.0 ** 60, 1e-6), (1.0, 1e10), (2.0 ** 60, 1.0), (3.0, 0.5)):
        h, hv = _f32(np.full(n, dent))
        fwd = losses.token_logprob(mx, _i32(t), inv_temperature=s)
        got = _np(losses.token_logprob_backward(mx, _i32(t), fwd, g, h, inv_temperature=s,
                                                out=torch.empty(n, v, dtype=torch.float32, device="cuda:0")))
        with np.errstate(invalid="ignore", divide="ignore"):
            want = L.token_logprob_bwd(xv, t, s, gv, hv)
        assert np.isfinite(got).all(), (s, dent, np.argwhere(~np.isfinite(got))[:4])
        tol = 4 * s * _err(v, 100.0) * (np.abs(gv) + hv * (4 + 2 * np.log(v)))[:, None]
        assert (np.abs(got - want) <= tol).all(), (s, dent, np.abs(got - want).max())
        masked = np.isneginf(xv)
        masked[np.arange(n), t] = False
        assert not got[masked].any()


# ------------------------------------------------------------------ infinite terms of the policy loss
@pytest.mark.parametrize("b,s", [(1, 5), (3, 64), (40, 1000)])
def test_policy_loss_of_tokens_that_cannot_occur(b, s):
    """A counted token whose log-probability is -inf under the policy (or was under the old one): its KL terms are +inf,
    which the loss has only with a weight on them; nothing is NaN."""
    import torch
    from paper_2606_30634_amd import losses
    base = torch.full((b, s), -1.0, device="cuda:0")
    on = torch.ones(b, s, dtype=torch.bool, device="cuda:0")
    adv = torch.ones(b, device="cuda:0")
    at = s // 2
    for who in ("policy", "old", "reference"):
        lp, old, ref = base.clone(), base.clone(), base - 0.5
        {"policy": lp, "old": old, "reference": ref}[who][b - 1, at] = -torch.inf
        for kl in (0.0, 0.25):
            log(f"{who} kl {kl}")
            got = losses.policy_loss(lp, old, adv, on, ref_logp=ref, kl_coef=kl)
            with np.errstate(invalid="ignore", over="ignore"):
                want = L.policy_loss(_np(lp), _np(old), _np(adv), on.cpu().numpy(), ref=_np(ref), kl_coef=kl)
            assert not bool(got.loss.isnan()) and not bool(got.metrics.isnan().any()) and not bool(got.dlogp.isnan().any())
            for g, w in ((got.loss, np.array([want["loss"]])), (got.metrics, want["metrics"]), (got.dlogp, want["dlogp"])):
                g = _np(g)
                fin = np.isfinite(w)
                assert (g[~fin] == w[~fin]).all() and (np.abs(g[fin] - w[fin]) <= 32 * U * (1 + np.abs(w[fin]))).all(), (who, kl, g, w)


# ------------------------------------------------------------------ many rows
@pytest.mark.parametrize("v", [1, 2])
def test_head_of_millions_of_unaligned_rows(v):
    """Rows of one or two tokens, a chunk of them far longer than it is wide."""
    import torch
    from paper_2606_30634_amd import losses
    n = 9_000_001
    x = torch.linspace(-4, 4, n, device="cuda:0").bfloat16().view(n, 1)
    w = torch.tensor([[1.0], [-0.5]], device="cuda:0").bfloat16()[:v].contiguous()
    t = torch.arange(n, device="cuda:0", dtype=torch.int32) % v
    got = losses.head_logprob(x, w, t)
    z = x.double() @ w.double().t()
    want = torch.log_softmax(z, 1).gather(1, t.long().view(n, 1)).view(n)
    assert float((got.logp.double() - want).abs().max()) <= 64 * U * 7


# ------------------------------------------------------------------ small gradients of the preference loss
@pytest.mark.parametrize("pairs,s", [(40, 3), (300, 2), (600, 20), (40, 5000)])
@pytest.mark.parametrize("smoothing", [0.0, 1.0])
def test_preference_gradient_of_pairs_far_apart(pairs, s, smoothing):
    """With all weight on one side the gradient of a pair that is far on it is beta sigmoid(-|h|), 10^-17 of the others'
    and as exact relatively: a rounding of the double and one of the result, 2 u with the scale's."""
    import torch
    from paper_2606_30634_amd import losses
    h = np.linspace(-40, 40, pairs)
    lp = np.zeros((2 * pairs, s))
    lp[:pairs, 0] = h
    t, v = _f32(lp)
    on = torch.ones(2 * pairs, s, dtype=torch.bool, device="cuda:0")
    got = losses.preference_loss(t, on, beta=1.0, label_smoothing=smoothing)
    want = L.preference_loss(v, np.ones((2 * pairs, s), bool), beta=1.0, label_smoothing=smoothing)
    for name in ("dlogp", "pair_loss"):
        d = np.abs(_np(getattr(got, name)) - want[name])
        assert (d <= 2 * U * np.abs(want[name])).all(), (name, (d / np.abs(want[name])).max() / U)
