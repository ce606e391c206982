"""Attention over key ranges at the ends of its arguments: shared rows (strides of 0), the largest and smallest caps, scales,
positions and range ends.  Bounds as in test_gpu_attention.py."""
import numpy as np
import pytest

from gpu_common import log
from oracle import attention as A
from test_gpu_attention import _case, _check_backward, _check_forward, _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("Sq,Sk", [(150, 150), (2, 600)])
def test_shared_rows(Sq, Sk, hd, bf16):
    """Inputs of strides 0 over sequences, rows or heads give what copies of them give."""
    import torch
    from paper_2606_30634_amd import attention as T
    log(f"Sq {Sq} Sk {Sk} hd {hd} bf16 {bf16}")
    B, H, KV = 3, 4, 2
    dt = torch.bfloat16 if bf16 else torch.float32
    g = torch.Generator(device="cuda:0").manual_seed(hd + Sk)
    new = lambda *s: torch.randn(*s, generator=g, device="cuda:0").to(dt)  # noqa: E731
    full = dict(q=(B, Sq, H, hd), k=(B, Sk, KV, hd), v=(B, Sk, KV, hd), do=(B, Sq, H, hd))
    for shared in (dict(k=0, v=0), dict(q=1, do=1), dict(k=2, v=2, q=2), dict(v=1), dict(q=0, do=2)):
        x = {n: new(*s) for n, s in full.items()}
        for n, d in shared.items():
            s = list(full[n])
            s[d] = 1
            x[n] = new(*s).expand(*full[n])
        c = {n: t.contiguous() for n, t in x.items()}
        f, fc = (T.attention(t["q"], t["k"], t["v"], softcap=5.0, keep_f32=bf16) for t in (x, c))
        assert torch.equal(f.o, fc.o) and torch.equal(f.lse, fc.lse)
        for a, b in zip(T.attention_backward(x["q"], x["k"], x["v"], f, x["do"], softcap=5.0),
                        T.attention_backward(c["q"], c["k"], c["v"], fc, c["do"], softcap=5.0)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("cap,scale,qexp", [(2.0 ** -60, 0.125, 0), (2.0 ** 100, 0.125, 0), (0.0, 2.0 ** 60, -60), (3.0, 2.0 ** 60, -60),
                                            (0.0, 2.0 ** -60, 0), (2.0 ** -60, 2.0 ** 60, 0), (2.0 ** 60, 2.0 ** -60, 0)])
def test_extreme_caps_and_scales(cap, scale, qexp, hd, bf16):
    log(f"cap {cap} scale {scale} hd {hd} bf16 {bf16}")
    x, how, rng, ref = _case(31, 2, 90, 90, 2, 1, hd, bf16, "documents", cap=cap, qstd=2.0 ** qexp)
    how["scale"], ref["scale"] = scale, scale
    with np.errstate(over="ignore"):  # the oracle's cosh of scores of 2^60 caps and more: a slope of 0
        f = _check_forward(x, how, rng, ref, bf16, bf16)
        _check_backward(x, how, rng, ref, bf16, f)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("Sq", [3, 140])
def test_extreme_positions_and_ranges(Sq, bf16):
    """Positions at both ends of int32, and ranges that end there."""
    log(f"Sq {Sq} bf16 {bf16}")
    lo, hi = -2 ** 31, 2 ** 31 - 1
    B, Sk, hd = 4, 160, 64
    first = np.array([lo, hi, 10, -1])
    x, how, _, ref = _case(32, B, Sq, Sk, 2, 1, hd, bf16, "causal")
    how["q_start"], ref["q_start"] = _i32(first), first
    rng = A.causal_ranges(B, Sq, Sk, first)
    f = _check_forward(x, how, rng, ref, bf16, bf16)
    _check_backward(x, how, rng, ref, bf16, f)
    r = np.random.default_rng(1)
    start, end = r.choice([lo, -1, 0, 5, Sk - 1, Sk, hi], size=(2, B, Sq))
    how.update(key_start=_i32(start), key_end=_i32(end))
    rng = np.maximum(start, 0), np.minimum(end, Sk)
    f = _check_forward(x, how, rng, ref, bf16, bf16)
    _check_backward(x, how, rng, ref, bf16, f)
