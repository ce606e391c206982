"""A stage whose blocks are a variant (stage_set_variant): packed documents, capped and biased scores, dropout, against
the float64 oracle of such a block, and against the plain stage where the variant changes nothing.  Bars: those of the
plain stage's parity tests, norm-wise per tensor: bf16 2e-2; fp32 1e-4 (its losses' bar, for sums of up to 512 terms)."""
import numpy as np
import pytest

import datagen
from gpu_common import hp_of, log, rel, shape_of, to_device
from oracle import attention as A
from oracle import model, ops

pytestmark = pytest.mark.gpu

BASE = dict(n_blocks=2, n_heads=4, n_kv_heads=2, d_ffn=256, vocab=0, first_stage=False, last_stage=False, tie_embedding=False,
            micro_batch=2, max_inflight=2)
F32 = datagen.TINY.with_(name="f32-middle", d_model=128, head_dim=32, seq_len=96, dtype="f32", **BASE)
F64 = datagen.TINY.with_(name="bf16-64", d_model=256, head_dim=64, seq_len=160, dtype="bf16", **BASE)
F128 = datagen.TINY.with_(name="bf16-128", d_model=512, head_dim=128, seq_len=200, dtype="bf16", **BASE)
HD32 = datagen.TINY.with_(name="bf16-32", d_model=128, head_dim=32, seq_len=77, dtype="bf16", **BASE)
STAGES = pytest.mark.parametrize("w", [F32, HD32, F64, F128], ids=lambda w: w.name)
FULL = dict(softcap=2.0, dropout=0.25, seed=2 ** 63 + 17, offset=2 ** 33 + 5, documents=True)


def _stage(w):
    from paper_2606_30634_amd.stage import Stage
    st = Stage(shape_of(w), "cuda:0")
    st.load_master(datagen.init_params(w))
    return st


def _documents(w, seed=0):
    r = np.random.default_rng(seed)
    cut = np.sort(r.integers(1, w.seq_len, size=(w.micro_batch, 3)), 1)
    ids = (np.arange(w.seq_len)[None, :, None] >= cut[:, None, :]).sum(2)
    ids = np.where(ids == 3, -1, ids).astype(np.int32)
    flags = np.zeros(ids.shape, np.uint8)
    for b in range(w.micro_batch):
        for d in range(3):
            at = np.nonzero(ids[b] == d)[0]
            flags[b, at[:len(at) // 3]] = 1
    return ids, flags


def _slopes(w):
    return (2.0 ** (-8.0 * (np.arange(w.n_heads) + 1) / w.n_heads)).astype(np.float32)


class Ref:
    """The variant's blocks in float64."""

    def __init__(self, w, ids, flags, slopes, softcap=0.0, dropout=0.0, seed=0, offset=0, documents=False):
        self.w, self.cap, self.p, self.seed, self.offset = w, softcap, dropout, seed, offset
        self.slopes = None if slopes is None else slopes.astype(np.float64)
        self.rng = A.key_ranges(ids, flags) if documents else A.causal_ranges(w.micro_batch, w.seq_len, w.seq_len)
        self.params = {k: v.astype(np.float64) for k, v in datagen.init_params(w).items()}

    def _drop(self, x, at):
        if not self.p:
            return x
        keep, f = A.dropout_keep(*x.shape, self.p, self.seed, at)
        return np.where(keep, x * f, 0.0)

    def step(self, inp):
        w, kw = self.w, dict(cap=self.cap, slopes=self.slopes)
        B, s, d, H, KV, hd = w.micro_batch, w.seq_len, w.d_model, w.n_heads, w.n_kv_heads, w.head_dim
        x = inp["x_in"].astype(np.float64).reshape(B * s, d)
        saves, at = [], self.offset
        for i in range(w.n_blocks):
            p = model._blk(self.params, i)
            n1, r1 = ops.rmsnorm_fwd(x, p["attn_norm"], w.rms_eps)
            q, k = (ops.rope_apply((n1 @ p[m].T).reshape(B, s, h, hd), w.rope_theta) for m, h in (("wq", H), ("wk", KV)))
            v = (n1 @ p["wv"].T).reshape(B, s, KV, hd)
            o = A.attention(q, k, v, *self.rng, **kw)[0].reshape(B * s, H * hd)
            h = x + self._drop(o @ p["wo"].T, at + 2 * i)
            n2, r2 = ops.rmsnorm_fwd(h, p["ffn_norm"], w.rms_eps)
            a, b = n2 @ p["wgate"].T, n2 @ p["wup"].T
            z = ops.swiglu_fwd(a, b)
            saves.append((x, n1, r1, q, k, v, o, h, n2, r2, a, b, z))
            x = h + self._drop(z @ p["wdown"].T, at + 2 * i + 1)
        y, g = x, {}
        dy = inp["dy"].astype(np.float64).reshape(B * s, d)
        for i in reversed(range(w.n_blocks)):
            p = model._blk(self.params, i)
            x, n1, r1, q, k, v, o, h, n2, r2, a, b, z = saves[i]
            e = f"blk{i}."
            dz, g[e + "wdown"] = ops.linear_bwd(self._drop(dy, at + 2 * i + 1), z, p["wdown"])
            da, db = ops.swiglu_bwd(dz, a, b)
            dg, g[e + "wgate"] = ops.linear_bwd(da, n2, p["wgate"])
            du, g[e + "wup"] = ops.linear_bwd(db, n2, p["wup"])
            dn, g[e + "ffn_norm"] = ops.rmsnorm_bwd(dg + du, h, r2, p["ffn_norm"])
            dh = dy + dn
            do, g[e + "wo"] = ops.linear_bwd(self._drop(dh, at + 2 * i), o, p["wo"])
            dq, dk, dv = A.attention_bwd(q, k, v, do.reshape(B, s, H, hd), *self.rng, **kw)
            dq, dk = (ops.rope_apply(t, w.rope_theta, inverse=True) for t in (dq, dk))
            dn = 0
            for m, t in (("wq", dq), ("wk", dk), ("wv", dv)):
                dx, g[e + m] = ops.linear_bwd(t.reshape(B * s, -1), n1, p[m])
                dn = dn + dx
            dx, g[e + "attn_norm"] = ops.rmsnorm_bwd(dn, x, r1, p["attn_norm"])
            dy = dh + dx
        self.offset += 2 * w.n_blocks if round(self.p * 65536) else 0
        return y, g, dy


def _run(st, w, inp, slot=0, step=0):
    """(y, gradients of this microbatch alone on a fresh step, dx)"""
    import torch
    dev = torch.device("cuda:0")
    d = to_device(inp, w, dev)
    dt = torch.bfloat16 if w.dtype == "bf16" else torch.float32
    y, dx = (torch.full((w.micro_batch, w.seq_len, w.d_model), float("nan"), dtype=dt, device=dev) for _ in range(2))
    st.forward(slot, step, x_in=d["x_in"], y_out=y)
    st.backward(slot, dy=d["dy"], dx_out=dx)
    torch.cuda.synchronize()
    names = list(datagen.init_params(w))
    return y, {n: st.view(f"grad0.{n}").clone() for n in names}, dx


def _np(t):
    return t.double().cpu().numpy()


@STAGES
@pytest.mark.parametrize("kind", ["all", "documents", "scores", "dropout"])
def test_blocks_against_the_oracle(w, kind):
    import torch
    log(f"{w.name} {kind}")
    how = {"all": FULL, "documents": dict(documents=True), "scores": dict(softcap=2.0), "dropout": dict(dropout=0.5, seed=3)}[kind]
    ids, flags = _documents(w)
    slopes = _slopes(w) if kind in ("all", "scores") else None
    ref = Ref(w, ids, flags if kind == "all" else None, slopes, **how)
    st = _stage(w)
    st.set_variant(slopes=None if slopes is None else torch.from_numpy(slopes).to("cuda:0"), **how)
    bar = 2e-2 if w.dtype == "bf16" else 1e-4
    total = None
    for n, slot in ((0, 0), (1, 1)):  # the second forward draws other masks; its gradient is added
        if how.get("documents"):
            st.set_documents(slot, torch.from_numpy(ids).to("cuda:0"), torch.from_numpy(flags).to("cuda:0") if kind == "all" else None)
        inp = datagen.step_inputs(w, 0, n)
        y, g, dx = _run(st, w, inp, slot)
        ry, rg, rdx = ref.step(inp)
        total = rg if total is None else {k: total[k] + rg[k] for k in rg}
        shape = (w.micro_batch * w.seq_len, w.d_model)
        assert rel(_np(y).reshape(shape), ry) < bar and rel(_np(dx).reshape(shape), rdx) < bar
        for k in total:
            assert rel(_np(g[k]).reshape(total[k].shape), total[k]) < bar, k
    st.close()


@STAGES
def test_a_variant_of_nothing_and_back(w):
    """A variant without any change gives the plain stage's results up to rounding, and the plain stage is bit for bit
    itself after it."""
    log(w.name)
    inp = datagen.step_inputs(w, 0)
    st = _stage(w)
    plain = _run(st, w, inp)
    st.close()
    st = _stage(w)
    st.set_variant()
    same = _run(st, w, inp)
    st.close()
    bar = 2e-2 if w.dtype == "bf16" else 1e-5
    for a, b in [(plain[0], same[0]), (plain[2], same[2])] + [(plain[1][k], same[1][k]) for k in plain[1]]:
        assert rel(_np(b), _np(a)) < bar
    st = _stage(w)
    st.set_variant(**dict(FULL, documents=False))
    st.clear_variant()
    again = _run(st, w, inp)
    st.close()
    import torch
    for a, b in [(plain[0], again[0]), (plain[2], again[2])] + [(plain[1][k], again[1][k]) for k in plain[1]]:
        assert torch.equal(a, b)


def test_interleaved_microbatches_and_updates():
    """1F1B with two microbatches in flight, each with its own documents and masks, and delayed updates: the same as one
    after another, bit for bit, in every overlap mode."""
    import torch
    w = F64
    log(w.name)
    hp = hp_of(w)
    docs = [tuple(torch.from_numpy(t).to("cuda:0") for t in _documents(w, m)) for m in range(2)]
    results = []
    for order, mode in (("FFBB", 0), ("FFBB", 1), ("FFBB", 2), ("FBFB", 0)):
        st = _stage(w)
        st.set_variant(**FULL)
        if mode:
            st.set_update_overlap(mode)
        for t in range(3):
            micro = [to_device(datagen.step_inputs(w, t, m), w, torch.device("cuda:0")) for m in range(2)]
            if mode:
                st.update(t, hp)
            for m in range(2):
                st.set_documents(m, *docs[m])
            f = b = 0
            for c in order:
                if c == "F":
                    st.forward(f, t, x_in=micro[f]["x_in"])
                    f += 1
                else:
                    st.backward(b, dy=micro[b]["dy"], microbatches_per_step=2)
                    b += 1
            if not mode:
                st.update(t, hp)
        st.join_update()
        torch.cuda.synchronize()
        results.append(st.view("flat.master").clone())
        st.close()
    for r in results[1:]:
        assert torch.equal(r, results[0])


def test_refusals():
    import torch
    from paper_2606_30634_amd import binding as B
    w = F64
    log(w.name)
    st = _stage(w)
    inp = to_device(datagen.step_inputs(w, 0), w, torch.device("cuda:0"))
    ids, flags = (torch.from_numpy(t).to("cuda:0") for t in _documents(w))
    for bad in (dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=float("inf")), dict(dropout=1.0), dict(dropout=-0.1)):
        with pytest.raises(B.StageError) as e:
            st.set_variant(**bad)
        assert e.value.code == B.STAGE_EINVAL
    v = B.StageVariant(0.0, None, 0.0, 0, 0, 1)
    n = B.stage_variant_bytes(st.handle, v)
    ws = torch.empty(n + 512, dtype=torch.uint8, device="cuda:0")
    p = (ws.data_ptr() + 255) // 256 * 256
    for args, code in (((None, n), B.STAGE_EINVAL), ((p + 16, n), B.STAGE_EINVAL), ((p, n - 1), B.STAGE_ENOSPACE)):
        with pytest.raises(B.StageError) as e:
            B.stage_set_variant(st.handle, v, *args)
        assert e.value.code == code
    with pytest.raises(ValueError):
        st.set_variant(slopes=torch.ones(3, device="cuda:0"))

    def refused(f, code=B.STAGE_ESTATE):
        with pytest.raises(B.StageError) as e:
            f()
        assert e.value.code == code

    refused(lambda: st.set_documents(0, ids))  # no variant
    st.set_variant(softcap=1.0)
    refused(lambda: st.set_documents(0, ids))  # a variant without documents
    st.set_variant(documents=True)
    refused(lambda: st.forward(0, 0, x_in=inp["x_in"]))  # documents not set
    refused(lambda: st.set_documents(2, ids), B.STAGE_EINVAL)
    for call in (lambda: st.set_documents(0, ids.long()), lambda: st.set_documents(0, ids[:1]), lambda: st.set_documents(0, ids, ids)):
        with pytest.raises(ValueError):
            call()
    st.set_documents(0, ids, flags)
    st.forward(0, 0, x_in=inp["x_in"])
    refused(lambda: st.set_variant(softcap=1.0))  # a backward is pending
    refused(lambda: st.clear_variant())
    refused(lambda: st.set_documents(0, ids))
    st.backward(0, dy=inp["dy"])
    st.clear_variant()
    st.close()


def test_packed_fine_tuning():
    """Answers packed in rows, trained through their log-probabilities: those of an answer are what they are alone in a
    row (up to bf16 rounding), scoring without dropout agrees with the forward, and the losses' gradients run back."""
    import torch
    from paper_2606_30634_amd import losses
    w = datagen.LAST.with_(name="last", n_blocks=2, d_model=256, n_heads=4, n_kv_heads=2, head_dim=64, d_ffn=512, vocab=1003,
                           seq_len=128, micro_batch=2, max_inflight=1)
    log(w.name)
    st = _stage(w)
    inp = to_device(datagen.step_inputs(w, 0), w, torch.device("cuda:0"))
    ids = torch.full((2, 128), -1, dtype=torch.int32, device="cuda:0")
    ids[:, :50], ids[:, 50:110] = 0, 1
    targets = torch.where(ids >= 0, inp["targets"], -1)
    lp, ent, score, alone = (torch.zeros(2, 128, device="cuda:0") for _ in range(4))
    st.set_variant(softcap=30.0, documents=True)
    st.set_documents(0, ids)
    st.score_logprob(0, 0, targets, score, x_in=inp["x_in"])
    st.forward_logprob(0, 0, targets, lp, x_in=inp["x_in"], entropy=ent)
    bar = 2.0 ** -6  # a few bf16 roundings along the residual stream, logits of size about 1
    assert float((score - lp).abs().max()) < bar
    out = losses.policy_loss(lp, lp.clone(), torch.ones(2, device="cuda:0"), ids >= 0, entropy=ent, entropy_coef=0.01)
    st.backward_logprob(0, out.dlogp, out.dentropy)
    g = st.view("grad0.blk0.wq").clone()
    assert bool(torch.isfinite(g).all()) and bool((g != 0).any())
    # the second answer moved to the front of its row, where it is alone
    x2 = inp["x_in"].clone()
    x2[:, :60] = inp["x_in"][:, 50:110]
    ids2 = torch.full_like(ids, -1)
    ids2[:, :60] = 7
    t2 = torch.full_like(targets, -1)
    t2[:, :60] = targets[:, 50:110]
    st.set_documents(0, ids2)
    st.score_logprob(0, 0, t2, alone, x_in=x2)
    assert float((alone[:, :60] - score[:, 50:110]).abs().max()) < bar
    # NaN in the padding's activations reaches no token that counts
    x3 = inp["x_in"].clone()
    x3[:, 110:] = float("nan")
    st.set_documents(0, ids)
    st.score_logprob(0, 0, targets, alone, x_in=x3)
    assert bool((alone[:, :110] == score[:, :110]).all())
    # with dropout the forward differs, its score does not
    st.set_variant(softcap=30.0, documents=True, dropout=0.1, seed=5)
    st.set_documents(0, ids)
    st.score_logprob(0, 0, targets, alone, x_in=inp["x_in"])
    assert bool((alone == score).all())
    st.forward_logprob(0, 0, targets, alone, x_in=inp["x_in"])
    assert not bool((alone == lp).all())
    st.close()
