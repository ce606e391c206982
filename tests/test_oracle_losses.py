"""Pins of the oracle's log-probability and loss functions: definitions on small numbers, and every gradient
against central differences in float64."""
import numpy as np
import pytest

from oracle import losses as L


def _diff(f, x, eps=1e-6):
    """Central differences of the scalar f at x."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + eps
        hi = f()
        x[i] = keep - eps
        g[i] = (hi - f()) / (2 * eps)
        x[i] = keep
    return g


def test_logprob_by_hand():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.1, 0.2, 0.7]])) + 3.0
    logp, ent, stats = L.token_logprob(x, np.array([0, 2]), 1.0)
    assert np.allclose(np.exp(logp), [0.5, 0.7], rtol=1e-14)
    assert np.allclose(ent, [1.5 * np.log(2), -(0.1 * np.log(0.1) + 0.2 * np.log(0.2) + 0.7 * np.log(0.7))], rtol=1e-13)
    assert np.allclose(stats[:, 0], x.max(1))
    # a masked token takes no probability; a row of nothing else has no distribution
    x[0, 0] = -np.inf
    x[1] = -np.inf
    logp, ent, _ = L.token_logprob(x, np.array([1, 2]), 2.0)
    assert np.allclose([logp[0], ent[0]], [-np.log(2), np.log(2)]) and logp[1] == -np.inf and ent[1] == 0
    assert not np.any(L.token_logprob(x, np.array([-1, 3]), 1.0)[0])


@pytest.mark.parametrize("s", [1.0, 1.7])
def test_logprob_gradient(s):
    r = np.random.default_rng(1)
    x, t = r.normal(size=(4, 6)) * 2, np.array([1, -1, 5, 0])
    g, h = r.normal(size=4), r.normal(size=4)

    def f():
        logp, ent, _ = L.token_logprob(x, t, s)
        return np.sum(g * logp + h * ent)
    assert np.allclose(L.token_logprob_bwd(x, t, s, g, h), _diff(f, x), atol=1e-8)


@pytest.mark.parametrize("reduction,norm", [("token", 0.0), ("sequence", 0.0), ("token", 5.0), ("sequence", 3.0)])
def test_policy_gradient(reduction, norm):
    r = np.random.default_rng(2)
    logp = -np.abs(r.normal(size=(3, 7)))
    old, ref, ent = logp + 0.3 * r.normal(size=(3, 7)), logp + 0.5 * r.normal(size=(3, 7)), np.abs(r.normal(size=(3, 7)))
    adv, mask = r.normal(size=(3, 7)), (r.random((3, 7)) < 0.6)
    mask[1] = False
    kw = dict(clip_low=0.2, clip_high=0.3, kl_coef=0.7, entropy_coef=0.4, reduction=reduction, norm=norm)

    def f():
        return L.policy_loss(logp, old, adv, mask, ref=ref, entropy=ent, **kw)["loss"]
    out = L.policy_loss(logp, old, adv, mask, ref=ref, entropy=ent, grad_scale=2.0, **kw)
    assert 0 < out["metrics"][3] and out["counts"].tolist() == [mask.sum(), 2]
    assert np.allclose(out["dlogp"], 2 * _diff(f, logp), atol=1e-8)
    assert np.allclose(out["dentropy"], 2 * _diff(f, ent), atol=1e-8)
    one = L.policy_loss(logp, logp, adv, mask)  # on the sampling policy: ratio 1, nothing clipped
    assert np.isclose(one["loss"], -adv[mask].mean()) and one["metrics"][5] == pytest.approx(1.0)
    none = L.policy_loss(logp, old, adv, np.zeros_like(mask))
    assert none["loss"] == 0 and not none["dlogp"].any()


def test_policy_of_a_token_that_cannot_occur():
    """e^d - 1 - d at d = +inf (the policy's log-probability is -inf) and at d = -inf (the reference's): infinite, and in
    the loss only with a weight."""
    logp, ref = np.full((1, 3), -1.0), np.full((1, 3), -1.5)
    for a in (logp, ref):
        keep, a[0, 1] = a[0, 1], -np.inf
        with np.errstate(invalid="ignore"):
            for kl, loss in ((0.5, np.inf), (0.0, -2 / 3 if a is logp else -1.0)):
                out = L.policy_loss(logp, np.full((1, 3), -1.0), np.ones(1), np.ones((1, 3)), ref=ref, kl_coef=kl)
                assert np.isclose(out["loss"], loss) and out["metrics"][1] == np.inf and not np.isnan(out["dlogp"]).any()
        a[0, 1] = keep


@pytest.mark.parametrize("kind,smoothing", [("sigmoid", 0.0), ("sigmoid", 0.2), ("hinge", 0.0), ("square", 0.0)])
@pytest.mark.parametrize("normalize", [False, True])
def test_preference_gradient(kind, smoothing, normalize):
    r = np.random.default_rng(3)
    logp, mask = -np.abs(r.normal(size=(8, 5))), r.random((8, 5)) < 0.7
    ref = logp + 0.5 * r.normal(size=(8, 5))
    mask[:, 0] = True
    mask[2] = False  # pair 2 has no chosen answer: it does not count
    kw = dict(kind=kind, beta=0.6, label_smoothing=smoothing, margin=0.1, length_normalize=normalize)

    def f():
        return L.preference_loss(logp, mask, ref=ref, **kw)["loss"]
    out = L.preference_loss(logp, mask, ref=ref, grad_scale=0.5, **kw)
    assert np.allclose(out["dlogp"], 0.5 * _diff(f, logp), atol=1e-8)
    assert out["counts"][0] == 3 and out["pair_loss"][2] == 0 and not out["dlogp"][[2, 6]].any()


def test_preference_by_hand():
    logp = np.array([[-1.0, -2.0], [-3.0, -9.0]])
    mask = np.array([[1, 1], [1, 0]])
    out = L.preference_loss(logp, mask, beta=0.5)  # equal scores: even odds
    assert np.isclose(out["loss"], np.log(2)) and np.allclose(out["dlogp"], [[-0.25, -0.25], [0.25, 0.0]])
    assert np.allclose(L.preference_loss(logp, mask, beta=0.5, kind="square")["loss"], 1.0)
    assert np.allclose(L.preference_loss(logp, mask, beta=0.5, length_normalize=True)["rewards"], [-0.75, -1.5])
