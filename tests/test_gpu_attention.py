"""Attention over key ranges and its key ranges on the GPU against the oracle in float64, at the sizes, masks, strides
and values where they can go wrong.

Tolerances count roundings, u = 2^-24.  A score is a sum of hd products (exact of the inputs) accumulated in fp32, its
scale, the cap (a tanh within 4 u relatively, two products) and the distance term: within
  (hd + 16) u (1 + sum |q||k| scale + |s|)  =: E (1 + ..), and 2^t of it adds 4 u.
lse takes the largest such error of its row, its own rounding and a sum of Sk positive terms: (Sk / 16 + 64) u (a thread
adds at most every sixteenth).  A probability then errs by its score's and its row's error, and, rounded to bf16, by 2^-8; kept as two
bf16 parts (keep_f32), by 2^-16.  o is rounded once more.  In the backward P and dS are rounded to bf16 (2^-8 each, of
bf16 inputs), delta carries the error of o (o_f32: as above; o in bf16: 2^-8), and each gradient is rounded once.
Probabilities below 2^-126 (fp32's least normal number) are 0: at most 2^14 of them in a sum, times factors below 2^12 here,
change it by less than 2^-100 =: TINY."""
import numpy as np
import pytest

from gpu_common import log
from oracle import attention as A

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -100
HALF = {False: 2.0 ** -24, True: 2.0 ** -8}


def _torch():
    import torch
    return torch


def _dev(a, bf16):
    """a on the device in its type, and the values it holds there"""
    torch = _torch()
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda:0")
    t = t.bfloat16() if bf16 else t
    return t, t.double().cpu().numpy()


def _i32(a):
    return _torch().tensor(np.asarray(a), dtype=_torch().int32, device="cuda:0")


def _np(t):
    return t.double().cpu().numpy()


def _within(name, got, want, tol):
    got = _np(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= tol + TINY)
    assert not bad.any(), (name, int(bad.sum()), got[bad][:3], want[bad][:3], np.broadcast_to(tol, want.shape)[bad][:3])


def _case(seed, B, Sq, Sk, H, KV, hd, bf16, mask="causal", cap=0.0, bias=False, qstd=1.0):
    """Inputs of one call: device tensors, their values, the call's keywords and the oracle's."""
    r = np.random.default_rng(seed)
    x = {}
    for n, s in (("q", (B, Sq, H, hd)), ("k", (B, Sk, KV, hd)), ("v", (B, Sk, KV, hd)), ("do", (B, Sq, H, hd))):
        x[n], x[n + "v"] = _dev(r.normal(size=s) * (qstd if n == "q" else 1.0), bf16)
    how, ref = dict(softcap=cap), dict(cap=cap)
    if bias:
        sl = np.float32(2.0) ** (-8.0 * (np.arange(H) + 1) / H).astype(np.float32)
        how["slopes"], ref["slopes"] = _torch().from_numpy(sl.astype(np.float32)).to("cuda:0"), sl.astype(np.float64)
    first = None
    if mask == "ragged":  # answers of different lengths in one cache
        first = r.integers(-Sq, Sk - Sq + 1, size=B)
        first[0] = Sk - Sq
        how["q_start"], ref["q_start"] = _i32(first), first
    if mask in ("causal", "ragged"):
        start, end = A.causal_ranges(B, Sq, Sk, first)
    else:
        if mask in ("documents", "prefix"):
            assert Sq == Sk
            cuts = np.sort(r.integers(0, Sk + 1, size=(B, 4)), 1)
            ids = (np.arange(Sk)[None, :, None] >= cuts[:, None, :]).sum(2)
            ids = np.where(ids == 4, -1, ids)
            flags = np.zeros((B, Sk), np.uint8)
            for b in range(B):
                for d in range(4):
                    at = np.nonzero(ids[b] == d)[0]
                    flags[b, at[:len(at) // 2]] = 1
            start, end = A.key_ranges(ids, flags if mask == "prefix" else None)
        elif mask == "random":  # any ranges, some empty, some outside the keys
            a = r.integers(-3, Sk + 4, size=(2, B, Sq))
            start, end = a.min(0), a.max(0)
            none = r.random((B, Sq)) < 0.2
            start, end = np.where(none, end + 1, start), np.where(none, start, end)
        elif mask == "window":
            end = np.arange(1, Sq + 1)[None, :].repeat(B, 0) + (Sk - Sq)
            start = np.maximum(0, end - 37)
        else:
            assert mask == "full"
            start, end = np.zeros((B, Sq), int), np.full((B, Sq), Sk)
        how["key_start"], how["key_end"] = _i32(start), _i32(end)
        start, end = np.maximum(start, 0), np.minimum(end, Sk)
    return x, how, (start, end), ref


def _check_forward(x, how, rng, ref, bf16, keep, only=slice(None)):
    from paper_2606_30634_amd import attention as T
    hd, Sk = x["qv"].shape[3], x["kv"].shape[1]
    f = T.attention(x["q"], x["k"], x["v"], keep_f32=keep, **how)
    o, lse = A.attention(x["qv"], x["kv"], x["vv"], *rng, **ref)
    prob = 0.0 if not bf16 else 2.0 ** -16 if keep else 2.0 ** -8
    bo, bl = A.attention_bounds(x["qv"], x["kv"], x["vv"], *rng, (hd + 16) * U, prob + (Sk / 16 + 64) * U, **ref)
    got, lse, bl, bo, o = _np(f.lse)[..., only], lse[..., only], bl[..., only], bo[:, only], o[:, only]
    assert ((got == -np.inf) == (lse == -np.inf)).all()
    fin = np.isfinite(lse)
    tol = bl + (Sk / 16 + 64) * U + 4 * U * np.abs(np.where(fin, lse, 0.0))
    assert (np.abs(np.where(fin, got - np.where(fin, lse, 0.0), 0.0)) <= tol).all(), np.abs(got - lse)[fin].max()
    _within("o", f.o[:, only], o, bo + HALF[bf16] * (np.abs(o) + bo))
    if f.o_f32 is not None:
        _within("o_f32", f.o_f32[:, only], o, bo + U * np.abs(o))
    else:
        assert not (keep and bf16)
    return f


def _check_backward(x, how, rng, ref, bf16, f, only=slice(None)):
    from paper_2606_30634_amd import attention as T
    hd, Sk, Sq = x["qv"].shape[3], x["kv"].shape[1], x["qv"].shape[1]
    got = T.attention_backward(x["q"], x["k"], x["v"], f, x["do"], **how)
    n = (max(Sk, Sq) / 16 + 64) * U
    rounded = HALF[bf16] if bf16 else 0.0
    delta = (hd + 16) * U + n + (0.0 if not bf16 else 2.0 ** -16 if f.o_f32 is not None else 2.0 ** -8)
    out = A.attention_bwd(x["qv"], x["kv"], x["vv"], x["dov"], *rng, **ref,
                          errors=((hd + 16) * U, rounded + 2 * n, rounded + 2 * n, delta))
    for name, g, w, b in zip(("dq", "dk", "dv"), got, out[:3], out[3:]):
        w, b = w[:, only], b[:, only]
        _within(name, g[:, only], w, b + HALF[bf16] * (np.abs(w) + b))
    return got


SHAPES = [  # B, Sq, Sk, H, KV, hd, mask
    (1, 1, 1, 1, 1, 32, "causal"), (2, 3, 3, 2, 1, 64, "causal"), (1, 33, 33, 4, 2, 128, "causal"), (2, 64, 64, 3, 3, 64, "documents"),
    (2, 129, 129, 2, 1, 128, "documents"), (1, 200, 200, 4, 1, 32, "prefix"), (2, 257, 257, 2, 2, 64, "prefix"),
    (1, 300, 300, 2, 1, 128, "prefix"), (3, 65, 131, 4, 2, 64, "random"), (2, 150, 77, 2, 1, 128, "random"), (1, 40, 300, 6, 3, 32, "window"),
    (1, 140, 333, 2, 2, 128, "window"), (2, 97, 97, 2, 1, 64, "full"), (2, 130, 60, 2, 2, 128, "causal"), (1, 255, 255, 8, 1, 128, "causal"),
    (1, 385, 385, 2, 1, 64, "causal")]


@pytest.mark.parametrize("form", ["plain", "cap", "bias", "both"])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,Sq,Sk,H,KV,hd,mask", SHAPES)
def test_forward_and_gradients(B, Sq, Sk, H, KV, hd, mask, bf16, form):
    log(f"B {B} Sq {Sq} Sk {Sk} heads {H}/{KV} hd {hd} {mask} bf16 {bf16} {form}")
    x, how, rng, ref = _case(Sq * 1009 + Sk, B, Sq, Sk, H, KV, hd, bf16, mask, cap=3.0 if form in ("cap", "both") else 0.0,
                             bias=form in ("bias", "both"), qstd=2.0)
    for keep in ((False, True) if bf16 else (False,)):
        f = _check_forward(x, how, rng, ref, bf16, keep)
        _check_backward(x, how, rng, ref, bf16, f)


FEW = [(1, 1, 2048, 4, 4, 128, "causal"), (3, 1, 1000, 8, 1, 64, "ragged"), (2, 5, 777, 6, 2, 32, "ragged"), (2, 16, 4100, 4, 1, 128, "ragged"),
       (1, 7, 7, 2, 2, 128, "causal"), (5, 2, 515, 2, 1, 128, "ragged"), (1, 1, 16385, 2, 1, 64, "causal"), (2, 3, 900, 16, 1, 128, "random"),
       (1, 9, 2500, 8, 1, 64, "window")]


@pytest.mark.parametrize("form", ["plain", "cap", "both"])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,Sq,Sk,H,KV,hd,mask", FEW)
def test_few_queries(B, Sq, Sk, H, KV, hd, mask, bf16, form):
    log(f"B {B} Sq {Sq} Sk {Sk} heads {H}/{KV} hd {hd} {mask} bf16 {bf16} {form}")
    x, how, rng, ref = _case(Sq * 31 + Sk, B, Sq, Sk, H, KV, hd, bf16, mask, cap=5.0 if form != "plain" else 0.0,
                             bias=form == "both", qstd=3.0)
    for keep in ((False, True) if bf16 else (False,)):
        f = _check_forward(x, how, rng, ref, bf16, keep)
    if Sk <= 4100:
        _check_backward(x, how, rng, ref, bf16, f)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("cap", [0.05, 0.5, 50.0, 1e4, 1e30])
def test_caps(cap, bf16, hd):
    """Scores far within the cap, around it and far beyond it (a tanh of 1, whose slope must not be noise)."""
    log(f"cap {cap} bf16 {bf16} hd {hd}")
    x, how, rng, ref = _case(11, 2, 70, 70, 2, 1, hd, bf16, "documents", cap=cap, qstd=4.0)
    f = _check_forward(x, how, rng, ref, bf16, bf16)
    _check_backward(x, how, rng, ref, bf16, f)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("few", [False, True])
def test_what_is_not_seen_has_no_influence(value, bf16, hd, few):
    """Padding, the rows of other documents and the unused end of a cache hold NaN or infinities."""
    torch = _torch()
    log(f"{value} bf16 {bf16} hd {hd} few {few}")
    B, H, KV = 2, 4, 2
    Sq, Sk = (3, 700) if few else (210, 210)
    x, how, rng, ref = _case(3, B, Sq, Sk, H, KV, hd, bf16, "ragged" if few else "documents", cap=4.0, bias=True)
    start, end = rng
    seen = np.zeros((B, Sk), bool)
    for b in range(B):
        for i in range(Sq):
            seen[b, start[b, i]:max(start[b, i], end[b, i])] = True
    key = torch.from_numpy(~seen).to("cuda:0")
    row = torch.from_numpy(start >= end).to("cuda:0")
    assert bool(key.any())
    for n in ("k", "v"):
        x[n][key] = value
    for n in ("q", "do"):
        x[n][row] = value
    f = _check_forward(x, how, rng, ref, bf16, bf16)  # against the oracle of the clean values
    _check_backward(x, how, rng, ref, bf16, f)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("bf16", [False, True])
def test_a_row_that_is_not_finite_stays_in_its_document(bf16, hd):
    """One document's keys, values, queries and output gradients hold NaN and infinities; its neighbours in the same
    tiles are what they are without it."""
    log(f"bf16 {bf16} hd {hd}")
    ids = np.repeat([0, 1, 2, 3], [50, 60, 37, 80])[None, :]
    start, end = A.key_ranges(ids)
    x, how, _, ref = _case(4, 1, 227, 227, 4, 2, hd, bf16, "full", cap=4.0)
    how["key_start"], how["key_end"] = _i32(start), _i32(end)
    other = ids[0] != 1
    x["v"][0, 70], x["k"][0, 80], x["q"][0, 90], x["do"][0, 100] = np.inf, np.nan, -np.inf, np.nan
    f = _check_forward(x, how, (start, end), ref, bf16, bf16, other)  # against the oracle of the clean values
    got = _check_backward(x, how, (start, end), ref, bf16, f, other)
    assert bool(_torch().isnan(f.o[0, 80:110]).any()) and all(bool(_torch().isnan(g[0, 50:110]).any()) for g in got)


def test_scores_that_overflow():
    """Scores of -inf are keys of no weight; a row of nothing else has lse -inf and o 0, as one that sees nothing."""
    torch = _torch()
    from paper_2606_30634_amd import attention as T
    for bf16 in (False, True):
        for hd in (32, 64, 128):
            for Sq in (1, 40):
                log(f"bf16 {bf16} hd {hd} Sq {Sq}")
                dt = torch.bfloat16 if bf16 else torch.float32
                q = torch.zeros(1, Sq, 1, hd, dtype=dt, device="cuda:0")
                k, v = torch.zeros(1, 90, 1, hd, dtype=dt, device="cuda:0"), torch.ones(1, 90, 1, hd, dtype=dt, device="cuda:0")
                q[..., 0], k[:, :, :, 0] = 1e30, -1e30
                k[:, 5, :, 0] = 0
                f = T.attention(q, k, v, key_start=_i32([[0] * Sq]), key_end=_i32([[90] * Sq]), scale=1.0)
                assert bool((f.o == 1).all()) and bool((f.lse == 0).all())
                f = T.attention(q, k, v, key_start=_i32([[6] * Sq]), key_end=_i32([[90] * Sq]), scale=1.0)
                assert bool((f.o == 0).all()) and bool((f.lse == -np.inf).all())
                g = T.attention_backward(q, k, v, f, torch.ones_like(q), key_start=_i32([[6] * Sq]), key_end=_i32([[90] * Sq]), scale=1.0)
                assert all(bool((t == 0).all()) for t in g)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_strides(hd, bf16):
    """Heads of one packed row, [B, H, S, hd] tensors and a cache longer than its keys give what copies of them give,
    and nothing outside the outputs is written."""
    torch = _torch()
    from paper_2606_30634_amd import attention as T
    log(f"hd {hd} bf16 {bf16}")
    B, S, H, KV = 2, 150, 4, 2
    x, how, rng, ref = _case(9, B, S, S, H, KV, hd, bf16, "documents", cap=4.0, bias=True)
    base = T.attention(x["q"], x["k"], x["v"], keep_f32=bf16, **how)
    grads = T.attention_backward(x["q"], x["k"], x["v"], base, x["do"], **how)

    def packed():
        buf = torch.full((B, S, H + 2 * KV, hd), float("nan"), dtype=x["q"].dtype, device="cuda:0")
        return buf, buf[:, :, :H], buf[:, :, H:H + KV], buf[:, :, H + KV:]

    def by_head(n):
        return torch.full((B, n, S, hd), float("nan"), dtype=x["q"].dtype, device="cuda:0").transpose(1, 2)

    def longer(n):
        return torch.full((B, S + 7, n + 1, hd), float("nan"), dtype=x["q"].dtype, device="cuda:0")[:, 3:3 + S, :n]

    for make in (lambda: packed()[1:], lambda: (by_head(H), by_head(KV), by_head(KV)), lambda: (longer(H), longer(KV), longer(KV))):
        q, k, v = make()
        for d, n in ((q, "q"), (k, "k"), (v, "v")):
            d.copy_(x[n])
        do = make()[0]
        do.copy_(x["do"])
        f = T.attention(q, k, v, keep_f32=bf16, **how)
        assert torch.equal(f.o, base.o) and torch.equal(f.lse, base.lse)
        out = make()
        T.attention_backward(q, k, v, f, do, out=out, **how)
        for a, b in zip(out, grads):
            assert torch.equal(a, b)
    # o (and o_f32) of another layout, as torch operations leave them
    far = base._replace(**{n: t.transpose(1, 2).contiguous().transpose(1, 2) for n, t in base._asdict().items()
                           if t is not None and n != "lse"})
    for a, b in zip(T.attention_backward(x["q"], x["k"], x["v"], far, x["do"], **how), grads):
        assert torch.equal(a, b)
    buf = longer(KV)
    whole = buf._base if buf._base is not None else buf
    T.attention_backward(x["q"], x["k"], x["v"], base, x["do"], out=(torch.empty_like(x["q"]), buf, torch.empty_like(x["v"])), **how)
    assert bool(torch.isnan(whole[:, :3]).all()) and bool(torch.isnan(whole[:, 3 + S:]).all()) and bool(torch.isnan(whole[:, :, KV:]).all())


@pytest.mark.parametrize("hd,bf16", [(128, True), (64, True), (64, False)])
def test_offsets_past_32_bits(hd, bf16):
    """Rows so far apart that their offsets pass 2^31 elements (and 2^32 bytes)."""
    torch = _torch()
    from paper_2606_30634_amd import attention as T
    log(f"hd {hd} bf16 {bf16}")
    S, H, KV, row = 300, 2, 1, 1 << 23
    dt = torch.bfloat16 if bf16 else torch.float32
    x, how, rng, ref = _case(21, 1, S, S, H, KV, hd, bf16, "causal")
    big = torch.empty(2 * S * row // 2, dtype=dt, device="cuda:0").view(1, S, row)
    far = {n: big[:, :, i * 512:i * 512 + h * hd].view(1, S, h, hd) for i, (n, h) in enumerate((("q", H), ("k", KV), ("v", KV), ("do", H)))}
    for n, t in far.items():
        t.copy_(x[n])
    a = T.attention(x["q"], x["k"], x["v"], **how)
    b = T.attention(far["q"], far["k"], far["v"], **how)
    assert torch.equal(a.o, b.o) and torch.equal(a.lse, b.lse)
    few = T.attention(far["q"][:, -2:], far["k"], far["v"])
    near = T.attention(x["q"][:, -2:], x["k"], x["v"])
    assert torch.equal(few.o, near.o)
    ga = T.attention_backward(x["q"], x["k"], x["v"], a, x["do"], **how)
    gb = T.attention_backward(far["q"], far["k"], far["v"], b, far["do"], **how)
    for s, t in zip(ga, gb):
        assert torch.equal(s, t)


def test_empty_sizes():
    torch = _torch()
    from paper_2606_30634_amd import attention as T
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device="cuda:0")  # noqa: E731
    for B, Sq, Sk in ((0, 4, 4), (2, 0, 5), (2, 5, 0), (0, 0, 0)):
        log(f"B {B} Sq {Sq} Sk {Sk}")
        q, k, v = z(B, Sq, 4, 64) + 1, z(B, Sk, 2, 64) + 1, z(B, Sk, 2, 64) + 1
        f = T.attention(q, k, v, keep_f32=True)
        assert f.o.shape == q.shape and not bool(f.o.any()) and bool((f.lse == -np.inf).all())
        out = tuple(torch.full_like(t, 7.0) for t in (q, k, v))
        T.attention_backward(q, k, v, f, q, out=out)
        assert not any(bool(t.any()) for t in out)


@pytest.mark.parametrize("bf16,hd", [(True, 128), (True, 64), (True, 32), (False, 64)])
def test_graphs_streams_and_repeats(bf16, hd):
    """Two captured passes sharing one workspace, replayed between eager work, and calls on another stream: the bits of
    the eager call every time."""
    torch = _torch()
    from paper_2606_30634_amd import attention as T, binding as B_
    log(f"bf16 {bf16} hd {hd}")
    cases = [_case(50, 2, 200, 200, 4, 2, hd, bf16, "documents", cap=5.0), _case(51, 2, 2, 1500, 4, 2, hd, bf16, "ragged", bias=True)]
    ws = torch.empty(256 << 20, dtype=torch.uint8, device="cuda:0")

    def run(x, how, w):
        f = T.attention(x["q"], x["k"], x["v"], keep_f32=bf16, workspace=w, **how)
        return [f.o, f.lse, *T.attention_backward(x["q"], x["k"], x["v"], f, x["do"], workspace=w, **how)]

    want = [run(x, how, None) for x, how, _, _ in cases]
    side = torch.cuda.Stream()
    graphs, outs = [], []
    for x, how, _, _ in cases:
        g = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(x, how, ws)
        torch.cuda.current_stream().wait_stream(side)
        with torch.cuda.graph(g):
            outs.append(run(x, how, ws))
        graphs.append(g)
    for rep in range(4):
        for g, o, w in zip(graphs, outs, want):
            for t in o:
                t.fill_(float("nan"))
            g.replay()
            if rep % 2:
                torch.cuda.synchronize()
            (torch.randn(300, 300, device="cuda:0") @ torch.randn(300, 300, device="cuda:0")).sum()
            for a, b in zip(o, w):
                assert torch.equal(a, b)
    with torch.cuda.stream(side):
        got = run(*cases[0][:2], None)
    side.synchronize()
    for a, b in zip(got, want[0]):
        assert torch.equal(a, b)


def test_captured_without_a_first_call():
    """Kernel variants no call has used before, captured at once, on the capture's own memory; eager calls of the same
    variants between the replays."""
    torch = _torch()
    from paper_2606_30634_amd import attention as T
    log("capture")
    for hd in (64, 128):
        for Sq, Sk in ((130, 130), (1, 3000)):
            x, how, _, _ = _case(60 + hd, 1, Sq, Sk, 2, 1, hd, True, "causal", cap=7.0, bias=True)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                f = T.attention(x["q"], x["k"], x["v"], keep_f32=True, **how)
                d = T.attention_backward(x["q"], x["k"], x["v"], f, x["do"], **how)
            want = None
            for _ in range(3):
                g.replay()
                torch.cuda.synchronize()
                got = [t.clone() for t in (f.o, f.lse, f.o_f32, *d)]
                e = T.attention(x["q"], x["k"], x["v"], keep_f32=True, **how)
                want = [e.o, e.lse, e.o_f32, *T.attention_backward(x["q"], x["k"], x["v"], e, x["do"], **how)]
                for a, b in zip(got, want):
                    assert torch.equal(a, b)


RANGE_ROWS = [(1, 1), (3, 2), (2, 7), (5, 64), (2, 513), (4, 2047), (3, 2048), (2, 2049), (2, 4097), (1, 9000)]


@pytest.mark.parametrize("prefix", [False, True])
@pytest.mark.parametrize("rows,length", RANGE_ROWS)
def test_key_ranges(rows, length, prefix):
    torch = _torch()
    from paper_2606_30634_amd import attention as T
    r = np.random.default_rng(rows * 7 + length)
    for mean in (1, 5, 300, 100000):
        log(f"rows {rows} length {length} prefix {prefix} mean {mean}")
        new = r.random((rows, length)) < 1.0 / mean
        ids = np.cumsum(new, 1) * 3 % 11
        ids = np.where(r.random((rows, 1)) < 0.5, ids, ids - 3).astype(np.int32)  # padding anywhere
        flags = (r.random((rows, length)) < 1 - 1.0 / (1 + mean / 2)).astype(np.uint8) * 255
        start, end = T.key_ranges(_i32(ids), prefix=torch.from_numpy(flags).to("cuda:0") if prefix else None)
        ws, we = _fast_ranges(ids, flags if prefix else None)
        if length <= 513:
            a, b = A.key_ranges(ids, flags if prefix else None)
            assert (a == ws).all() and (b == we).all()
        np.testing.assert_array_equal(start.cpu().numpy(), ws)
        np.testing.assert_array_equal(end.cpu().numpy(), we)


def _fast_ranges(ids, flags):
    """The oracle's ranges, document by document"""
    start, end = np.zeros(ids.shape, np.int32), np.zeros(ids.shape, np.int32)
    for b, row in enumerate(ids):
        cuts = [0, *(np.nonzero(np.diff(row))[0] + 1).tolist(), row.size]
        for lo, hi in zip(cuts[:-1], cuts[1:]):
            if row[lo] >= 0:
                start[b, lo:hi], end[b, lo:hi] = lo, np.arange(lo, hi) + 1
                if flags is not None:
                    off = np.nonzero(flags[b, lo:hi] == 0)[0]
                    n = lo + int(off[0]) if off.size else hi
                    end[b, lo:n] = n
    return start, end


def test_ranges_attention_and_gradient_together():
    """A packed batch as a training step uses it: ranges, forward, backward; each document as if it were alone."""
    torch = _torch()
    from paper_2606_30634_amd import attention as T
    for bf16 in (False, True):
        for hd in (32, 64, 128):
            log(f"bf16 {bf16} hd {hd}")
            lens = [100, 1, 63, 130]
            ids = torch.tensor(np.repeat([4, 0, 9, -1], lens)[None, :], dtype=torch.int32, device="cuda:0")
            x, _, _, _ = _case(77, 1, sum(lens), sum(lens), 4, 2, hd, bf16, "full")
            start, end = T.key_ranges(ids)
            f = T.attention(x["q"], x["k"], x["v"], key_start=start, key_end=end, keep_f32=bf16)
            g = T.attention_backward(x["q"], x["k"], x["v"], f, x["do"], key_start=start, key_end=end)
            at = 0
            for n in lens[:3]:
                part = {m: x[m][:, at:at + n].contiguous() for m in ("q", "k", "v", "do")}
                fa = T.attention(part["q"], part["k"], part["v"], keep_f32=bf16)
                ga = T.attention_backward(part["q"], part["k"], part["v"], fa, part["do"])
                for a, b in zip((f.o, *g), (fa.o, *ga)):
                    d = (a[:, at:at + n].float() - b.float()).abs().max()
                    # the tiles begin elsewhere: other partial sums, and a rounding that may fall to the other side.  And dS is
                    # a difference: of one token it is 0, as dP and delta are two sums of the same hd products, each
                    # within hd u sum |dO v| of the other, whatever their order; times scale |k| (|q|), over n queries of H heads.
                    noise = U * hd * hd * float(x["do"].abs().max() * x["v"].abs().max()) * hd ** -0.5 \
                        * float(torch.maximum(x["q"].abs().max(), x["k"].abs().max())) * n * 4
                    assert float(d) <= (2.0 ** -6 if bf16 else 2.0 ** -17) * float(b.float().abs().max()) + noise, (n, float(d))
                at += n
            assert not any(bool(t[:, at:].any()) for t in (f.o, *g))
