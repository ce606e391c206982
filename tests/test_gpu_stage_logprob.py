"""A last stage trained through log-probabilities: stage_forward_logprob / stage_backward_logprob /
stage_score_logprob with the losses on them, against the stage's own cross-entropy and the float64 oracle."""
import numpy as np
import pytest

import datagen
from gpu_common import hp_of, log, rel, shape_of, to_device
from oracle import losses as L
from oracle import model, ops

pytestmark = pytest.mark.gpu

TIED = datagen.TINY.with_(n_blocks=1, seq_len=32, micro_batch=2, max_inflight=2)
WIDE = datagen.LAST.with_(name="last", n_blocks=1, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ffn=512,
                          vocab=1003, seq_len=96, micro_batch=3, max_inflight=2)


def _stage(w, **kw):
    from paper_2606_30634_amd.stage import Stage
    st = Stage(shape_of(w, **kw), "cuda:0")
    st.load_master(datagen.init_params(w))
    return st


def _empty(w, n=1):
    import torch
    out = [torch.full((w.micro_batch, w.seq_len), 9.0, device="cuda:0") for _ in range(n)]
    return out if n > 1 else out[0]


def _oracle_logits(w, p0, inp):
    """Logits of one microbatch in float64, and the gradients of every parameter given dlogits."""
    p = {k: v.astype(np.float64) for k, v in p0.items()}
    x = ops.embed_fwd(p["embed"], inp["tokens"]) if w.first_stage else inp["x_in"].astype(np.float64)
    saves = []
    for i in range(w.n_blocks):
        x, sv = model.block_fwd(model._blk(p, i), x, w, np.float64)
        saves.append(sv)
    T = w.micro_batch * w.seq_len
    y = x.reshape(T, w.d_model)
    hf, r = ops.rmsnorm_fwd(y, p["final_norm"], w.rms_eps)
    W = p["embed" if w.tie_embedding else "head"]
    return hf @ W.T, (p, saves, y, hf, r, W)


def _oracle_grads(w, ctx, inp, dlogits):
    p, saves, y, hf, r, W = ctx
    g = {}
    dhf, dW = ops.linear_bwd(dlogits, hf, W)
    d, g["final_norm"] = ops.rmsnorm_bwd(dhf, y, r, p["final_norm"])
    d = d.reshape(w.micro_batch, w.seq_len, w.d_model)
    for i in reversed(range(w.n_blocks)):
        d, gb = model.block_bwd(model._blk(p, i), saves[i], d, w)
        g.update({f"blk{i}.{k}": v for k, v in gb.items()})
    g["embed" if w.tie_embedding else "head"] = dW
    if w.first_stage:
        de, _, _ = ops.embed_bwd(d, inp["tokens"], w.vocab)
        g["embed"] = g["embed"] + de
    return g, d


@pytest.mark.parametrize("w", [TIED, WIDE], ids=["f32-tied", "bf16-last"])
def test_logprobs_of_the_cross_entropy(w):
    """The mean of -logp is the stage's own loss, and its gradient (dlogp = -1/T) the stage's own gradient:
    the same logits, whose exponentials both take to about an ulp."""
    import torch
    st = _stage(w)
    inp = datagen.step_inputs(w, 0)
    d = to_device(inp, w, torch.device("cuda:0"))
    T = w.micro_batch * w.seq_len
    loss = torch.zeros(1, device="cuda:0")
    names = st.param_names()
    st.forward(0, 0, tokens=d.get("tokens"), x_in=d.get("x_in"), targets=d["targets"], loss=loss)
    st.backward(0)
    torch.cuda.synchronize()
    own = {n: st.view(f"grad0.{n}").double().cpu().numpy() for n in datagen.init_params(w)}
    st.close()
    st = _stage(w)
    lp, ent, score, sent = _empty(w, 4)
    kw = dict(tokens=d.get("tokens"), x_in=d.get("x_in"))
    st.score_logprob(1, 0, d["targets"], score, entropy=sent, **kw)
    st.forward_logprob(0, 0, d["targets"], lp, entropy=ent, **kw)
    st.backward_logprob(0, torch.full_like(lp, -1.0 / T))
    torch.cuda.synchronize()
    assert abs(float(loss) + float(lp.double().mean())) <= 1e-6 * abs(float(loss))
    # scoring takes the products of the same operands in another order: fp32 sums of d terms
    scale = float(lp.abs().max()) + 1
    assert float((score - lp).abs().max()) <= 2.0 ** -24 * (2 * w.d_model + 256) * scale
    assert float((sent - ent).abs().max()) <= 2.0 ** -24 * (2 * w.d_model + 256) * scale
    # bf16: dlogits round to bf16 on both sides, which an ulp of difference before can move by a step (2^-8)
    bar = 1e-5 if w.dtype == "f32" else 2.0 ** -8
    for n, g in own.items():
        e = rel(st.view(f"grad0.{n}").double().cpu().numpy(), g)
        log(f"{w.dtype} {n} {e:.2e}")
        assert e <= bar, (n, e)
    assert names
    st.close()


@pytest.mark.parametrize("w", [TIED, WIDE], ids=["f32-tied", "bf16-last"])
@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_step_against_the_oracle(w, kind):
    """Reference log-probabilities, the forward, a loss, the backward: log-probabilities, loss and every
    gradient against the float64 oracle; some targets ignored.  Bars: those of the stage's other parity
    tests, 1e-4 (fp32) and 2e-2 (bf16) of a tensor's norm."""
    import torch
    from paper_2606_30634_amd import losses
    if kind == "preference":
        w = w.with_(micro_batch=4)
    dev = torch.device("cuda:0")
    st = _stage(w)
    p0 = datagen.init_params(w)
    inp = datagen.step_inputs(w, 0)
    inp["targets"][0, :5] = -1
    inp["targets"][1, 7] = w.vocab
    d = to_device(inp, w, dev)
    r = np.random.default_rng(4)
    B, S = w.micro_batch, w.seq_len
    mask = (inp["targets"] >= 0) & (inp["targets"] < w.vocab) & (r.random((B, S)) < 0.8)
    s = 1.25
    lp, ent, ref = _empty(w, 3)
    kw = dict(tokens=d.get("tokens"), x_in=d.get("x_in"), inv_temperature=s)
    st.score_logprob(0, 0, d["targets"], ref, **kw)
    st.forward_logprob(0, 0, d["targets"], lp, entropy=ent, **kw)
    shift = torch.from_numpy((0.2 * r.normal(size=(B, S))).astype(np.float32)).to(dev)
    old, ref = lp + shift, ref - 0.5 * shift
    m = torch.from_numpy(mask).to(dev)
    adv = torch.from_numpy(r.normal(size=B).astype(np.float32)).to(dev)
    if kind == "policy":
        pk = dict(clip_low=0.25, clip_high=0.25, kl_coef=0.125, entropy_coef=0.0625)
        out = losses.policy_loss(lp, old, adv, m, ref_logp=ref, entropy=ent, **pk)
        dent = out.dentropy
    else:
        pk = dict(beta=0.5)
        out = losses.preference_loss(lp, m, ref_logp=ref, **pk)
        dent = None
    st.backward_logprob(0, out.dlogp, dent)
    torch.cuda.synchronize()
    x, ctx = _oracle_logits(w, p0, inp)
    t = inp["targets"].reshape(-1)
    want_lp, want_ent, _ = L.token_logprob(x, t, s)
    bar = 1e-4 if w.dtype == "f32" else 2e-2
    assert rel(lp.double().cpu().numpy().reshape(-1), want_lp) <= bar
    assert rel(ent.double().cpu().numpy().reshape(-1), want_ent) <= bar
    # the loss's gradients are the loss's own tests' matter: the chain back is held to them as they are
    dlogits = L.token_logprob_bwd(x, t, s, out.dlogp.double().cpu().numpy().reshape(-1),
                                  None if dent is None else dent.double().cpu().numpy().reshape(-1))
    grads, dx = _oracle_grads(w, ctx, inp, dlogits)
    for n in p0:
        e = rel(st.view(f"grad0.{n}").double().cpu().numpy().reshape(p0[n].shape), grads[n])
        log(f"{kind} {w.dtype} {n} {e:.2e}")
        assert e <= bar, (n, e)
    st.close()


def test_training_through_overlapped_updates():
    """Steps of score, forward, policy loss, backward and a delayed update in the overlap modes: the same
    numbers as without overlap (every read of a weight version is ordered before the update that overwrites
    it), and a step with a skipped microbatch in between."""
    import torch
    from paper_2606_30634_amd import losses
    w = WIDE
    runs = []
    for mode in (0, 1, 2):
        st = _stage(w)
        st.set_update_overlap(mode)
        lp, ref = _empty(w, 2)
        adv = torch.linspace(-1, 1, w.micro_batch, device="cuda:0")
        seen = []
        for t in range(5):
            d = to_device(datagen.step_inputs(w, t), w, torch.device("cuda:0"))
            st.update(t, hp_of(w)) if mode else None
            st.forward_logprob(0, t, d["targets"], lp, x_in=d["x_in"])
            # a read of the version after this step's last backward was issued, in the other slot
            out = losses.policy_loss(lp, lp, adv, torch.ones_like(lp, dtype=torch.bool))
            st.backward_logprob(0, out.dlogp)
            st.score_logprob(1, t, d["targets"], ref, x_in=d["x_in"])
            seen += [lp.clone(), ref.clone()]
            st.update(t, hp_of(w)) if not mode else None
        st.join_update()
        torch.cuda.synchronize()
        seen.append(st.view("flat.master").clone())
        runs.append(seen)
        st.close()
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


def test_order_and_arguments():
    import torch
    from paper_2606_30634_amd import binding as B
    w = WIDE
    st = _stage(w)
    d = to_device(datagen.step_inputs(w, 0), w, torch.device("cuda:0"))
    lp = _empty(w)
    loss = torch.zeros(1, device="cuda:0")

    def refused(code, f, *a, **k):
        with pytest.raises(B.StageError) as e:
            f(*a, **k)
        assert e.value.code == code, e.value
    refused(B.STAGE_ESTATE, st.backward_logprob, 0, lp)                                   # no forward yet
    refused(B.STAGE_EINVAL, st.forward_logprob, 0, 0, None, lp, x_in=d["x_in"])
    refused(B.STAGE_EINVAL, st.forward_logprob, 0, 0, d["targets"], None, x_in=d["x_in"])
    refused(B.STAGE_EINVAL, st.forward_logprob, 0, 0, d["targets"], lp)
    refused(B.STAGE_EINVAL, st.forward_logprob, 0, 0, d["targets"], lp, x_in=d["x_in"], inv_temperature=0.0)
    refused(B.STAGE_EINVAL, st.score_logprob, 2, 0, d["targets"], lp, x_in=d["x_in"])
    refused(B.STAGE_ESTATE, st.score_logprob, 0, 1, d["targets"], lp, x_in=d["x_in"])     # x_1 is not there
    st.forward_logprob(0, 0, d["targets"], lp, x_in=d["x_in"])
    refused(B.STAGE_ESTATE, st.forward_logprob, 0, 0, d["targets"], lp, x_in=d["x_in"])   # pending
    refused(B.STAGE_ESTATE, st.score_logprob, 0, 0, d["targets"], lp, x_in=d["x_in"])
    refused(B.STAGE_ESTATE, st.backward, 0)                                               # of the other kind
    refused(B.STAGE_EINVAL, st.backward_logprob, 0, None)
    refused(B.STAGE_EINVAL, st.backward_logprob, 0, lp, microbatches_per_step=0)
    st.forward(1, 0, x_in=d["x_in"], targets=d["targets"], loss=loss)
    refused(B.STAGE_ESTATE, st.backward_logprob, 1, lp)
    st.backward(1)
    st.backward_logprob(0, lp)
    torch.cuda.synchronize()
    st.close()
    mid = datagen.MID.with_(n_blocks=1, d_model=128, n_heads=2, n_kv_heads=2, head_dim=64, d_ffn=256, seq_len=64,
                            micro_batch=1)
    st = _stage(mid)
    x = torch.zeros(1, 64, 128, dtype=torch.bfloat16, device="cuda:0")
    t = torch.zeros(1, 64, dtype=torch.int32, device="cuda:0")
    refused(B.STAGE_EINVAL, st.forward_logprob, 0, 0, t, torch.zeros(1, 64, device="cuda:0"), x_in=x)
    refused(B.STAGE_EINVAL, st.score_logprob, 0, 0, t, torch.zeros(1, 64, device="cuda:0"), x_in=x)
    st.close()
