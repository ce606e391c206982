"""What the log-probability and loss operators refuse, through the C ABI and through the torch layer: every
refusal comes before anything touches a device, so this runs without one."""
import ctypes as C
import math

import pytest
import torch

from paper_2606_30634_amd import binding as B
from paper_2606_30634_amd import losses

P = 1 << 20  # an aligned address that is never read
Q = 1 << 40  # another, far from it


def _refused(fn, *args):
    with pytest.raises(B.StageError) as e:
        fn(*args)
    assert e.value.code == B.STAGE_EINVAL and B.last_error()


def _with(base, **kw):
    d = dict(base, **kw)
    return list(d.values())


FWD = dict(rows=4, vocab=100, logits=P, ld=100, bf=0, targets=P, s=1.0, logp=Q, ent=Q + 4096, stats=Q + 8192, ws=Q,
           nb=1 << 30, stream=None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(ld=99),
                                 dict(ld=(1 << 28) + 1), dict(logits=None), dict(logits=P + 2), dict(targets=None),
                                 dict(targets=P + 1), dict(logp=None), dict(ent=Q + 2), dict(stats=Q + 1), dict(s=0.0),
                                 dict(s=-1.0), dict(s=math.inf), dict(s=math.nan), dict(s=2.0 ** 61), dict(bf=1, logits=P + 1)])
def test_token_logprob_refuses(bad):
    _refused(B.token_logprob, *_with(FWD, **bad))


BWD = dict(rows=4, vocab=100, logits=P, ld=100, bf=0, targets=P, stats=P, ent=P, dlogp=P, dent=P, s=1.0, out=Q, ldo=100,
           obf=0, stream=None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(vocab=0), dict(ld=99), dict(ldo=99), dict(stats=None), dict(ent=None),
                                 dict(dlogp=None), dict(out=None), dict(out=Q + 2), dict(s=0.0), dict(logits=None),
                                 dict(out=P + 16), dict(out=P, ldo=101), dict(out=P, obf=1), dict(dent=P + 2)])
def test_token_logprob_backward_refuses(bad):
    _refused(B.token_logprob_backward, *_with(BWD, **bad))


HEAD = dict(rows=4, vocab=100, d=64, x=P, ldx=64, w=P, ldw=64, bf=1, targets=P, s=1.0, logp=Q, ent=Q + 4096,
            stats=Q + 8192, ws=Q, nb=1 << 30, stream=None)


@pytest.mark.parametrize("bad", [dict(d=0), dict(d=(1 << 20) + 1), dict(ldx=63), dict(ldw=63), dict(x=None), dict(w=None),
                                 dict(x=P + 1), dict(ldw=(1 << 24) + 1), dict(targets=None), dict(s=math.nan),
                                 dict(rows=-5), dict(vocab=0), dict(ws=None), dict(ws=Q + 16), dict(nb=8)])
def test_head_logprob_refuses(bad):
    _refused(B.head_logprob, *_with(HEAD, **bad))


POL = dict(seqs=64, len=1000, logp=P, old=P, ref=P, ent=P, adv=P, mask=P, hp=None, loss=Q, dlogp=Q, dent=Q + (1 << 20),
           metrics=Q, counts=Q, ws=Q, nb=1 << 30, stream=None)
POL_HP = dict(clip_low=0.2, clip_high=0.2, kl=0.1, ent=0.1, norm=0.0, gs=1.0, reduction=0, per_token=0)


@pytest.mark.parametrize("bad", [dict(seqs=-1), dict(len=-1), dict(seqs=1 << 31, len=1), dict(seqs=1 << 20, len=1 << 20),
                                 dict(logp=None), dict(old=None), dict(adv=None), dict(mask=None), dict(loss=None),
                                 dict(dlogp=None), dict(dent=None), dict(ent=None), dict(ref=None), dict(metrics=None),
                                 dict(counts=None), dict(counts=Q + 4), dict(logp=P + 2), dict(dlogp=P), dict(dent=P + 64),
                                 dict(dent=Q + 64), dict(ws=None), dict(nb=16), dict(ws=Q + 128),
                                 dict(hp=dict(clip_low=-0.1)), dict(hp=dict(clip_low=1.1)), dict(hp=dict(clip_high=-1.0)),
                                 dict(hp=dict(clip_high=math.inf)), dict(hp=dict(clip_low=math.nan)),
                                 dict(hp=dict(kl=math.nan)), dict(hp=dict(ent=math.inf)), dict(hp=dict(norm=-1.0)),
                                 dict(hp=dict(norm=math.inf)), dict(hp=dict(gs=math.nan)), dict(hp=dict(reduction=2))])
def test_policy_loss_refuses(bad):
    hp = B.PolicyHParams(*_with(POL_HP, **bad.pop("hp", {}) if isinstance(bad.get("hp"), dict) else {}))
    _refused(B.policy_loss, *_with(POL, **dict(bad, hp=hp)))


PREF = dict(pairs=64, len=1000, logp=P, ref=P, mask=P, hp=None, loss=Q, dlogp=Q, pair=Q, rewards=Q, metrics=Q, counts=Q,
            ws=Q, nb=1 << 30, stream=None)
PREF_HP = dict(beta=0.1, smoothing=0.0, margin=0.0, kind=0, normalize=0, norm=0.0, gs=1.0)


@pytest.mark.parametrize("bad", [dict(pairs=-1), dict(pairs=(1 << 24) + 1), dict(len=-1), dict(len=1 << 31),
                                 dict(pairs=1 << 24, len=1 << 20), dict(logp=None), dict(mask=None), dict(loss=None),
                                 dict(dlogp=None), dict(pair=None), dict(rewards=None), dict(metrics=None),
                                 dict(counts=None), dict(dlogp=P), dict(dlogp=P + 8), dict(ws=None), dict(nb=1),
                                 dict(hp=dict(beta=0.0)), dict(hp=dict(beta=-1.0)), dict(hp=dict(beta=math.inf)),
                                 dict(hp=dict(smoothing=-0.1)), dict(hp=dict(smoothing=1.5)), dict(hp=dict(kind=3)),
                                 dict(hp=dict(kind=1, smoothing=0.1)), dict(hp=dict(margin=math.nan)),
                                 dict(hp=dict(norm=-2.0)), dict(hp=dict(gs=math.inf))])
def test_preference_loss_refuses(bad):
    hp = B.PreferenceHParams(*_with(PREF_HP, **bad.pop("hp", {}) if isinstance(bad.get("hp"), dict) else {}))
    _refused(B.preference_loss, *_with(PREF, **dict(bad, hp=hp)))


def test_null_hparams():
    LIB = B.LIB
    null = C.POINTER(B.PolicyHParams)()
    assert LIB.policy_loss(*_with(POL, hp=null)) == B.STAGE_EINVAL
    assert LIB.preference_loss(*_with(PREF, hp=C.POINTER(B.PreferenceHParams)())) == B.STAGE_EINVAL


def test_workspace_bytes_of_refused_sizes():
    assert B.token_logprob_workspace_bytes(-1, 100) == 0 and B.head_logprob_workspace_bytes(4, 100, 0, 1) == 0
    assert B.policy_loss_workspace_bytes(1 << 20, 1 << 20) == 0 and B.preference_loss_workspace_bytes(1 << 25, 1) == 0
    assert B.token_logprob_workspace_bytes(0, 100) == 0


def test_no_rows_is_no_work():
    B.token_logprob(*_with(FWD, rows=0, logits=None, targets=None, logp=None, ws=None, nb=0))
    B.token_logprob_backward(*_with(BWD, rows=0, logits=None, out=None))
    B.head_logprob(*_with(HEAD, rows=0, x=None, w=None, ws=None, nb=0))


@pytest.mark.parametrize("call", [
    lambda f, i: losses.token_logprob(f(4, 10), i(4)),                       # not on a GPU
    lambda f, i: losses.token_logprob_backward(f(4, 10), i(4), losses.LogProb(), f(4)),
    lambda f, i: losses.head_logprob(f(4, 8), f(10, 8), i(4)),
    lambda f, i: losses.policy_loss(f(2, 8), f(2, 8), f(2), f(2, 8) > 0),
    lambda f, i: losses.preference_loss(f(2, 8), f(2, 8) > 0),
    lambda f, i: losses.token_logprob(f(4, 10).double(), i(4)),
    lambda f, i: losses.policy_loss(f(8), f(8), f(1), f(8) > 0),
    lambda f, i: losses.token_logprob(None, i(4)),
    lambda f, i: losses.policy_loss(None, f(2, 8), f(2), f(2, 8) > 0),
    lambda f, i: losses.preference_loss([[0.0]], f(2, 8) > 0)])
def test_torch_layer_refuses(call):
    with pytest.raises(ValueError):
        call(lambda *s: torch.zeros(*s), lambda n: torch.zeros(n, dtype=torch.int32))
