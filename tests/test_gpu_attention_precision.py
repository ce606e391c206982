"""What the forward of bf16 attention keeps of its weights where o is kept in fp32: 24 bits.

Every query sees two keys, one of score 0 and value 0, one of score -s (0 < s < 2) and value 1: o = p / (1 + p), p = exp(-s),
relative errors alone, u = 2^-24.  Scores are exact products; in log2 units they are off by 2 u |s| log2(e), so p by 2 u s + 2 u
(exp2 to one unit in the last place) <= 6 u; its three parts and their sum in fp32 by 4 u; sum, reciprocal, the shares' weights and
products by 6 u more: 16 u in all.  A cap adds its tanh, 2^-23 and three roundings of s: 10 u.  A p in two parts, 16 bits, is off by up to 128 u."""
import numpy as np
import pytest

from gpu_common import log

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def _inputs(B, Sq, Sk, H, KV, hd, seed=5):
    """(q, k, v, start, end, s [B, Sq]); q and k of one element, so that the scores are exact"""
    import torch
    r = np.random.default_rng(seed)
    dev, bf = "cuda:0", torch.bfloat16
    s = torch.from_numpy(r.uniform(0.05, 2.0, size=(B, Sk // 2)).astype(np.float32)).bfloat16()
    q, k, v = (torch.zeros(*n, hd, dtype=bf) for n in ((B, Sq, H), (B, Sk, KV), (B, Sk, KV)))
    q[..., 3] = 1.0
    k[:, 1::2, :, 3] = -s[:, :, None]
    v[:, 1::2] = 1.0
    at = torch.from_numpy(np.stack([r.permutation(Sk // 2)[:Sq] for _ in range(B)]).astype(np.int64))
    seen = torch.gather(s.double(), 1, at).numpy()
    start = (2 * at).int()
    return q.to(dev), k.to(dev), v.to(dev), start.to(dev), (start + 2).to(dev), seen


@pytest.mark.parametrize("cap", [0.0, 3.0])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("B,Sq,Sk,H,KV", [(2, 200, 400, 2, 1), (1, 385, 800, 2, 2), (40, 4, 400, 4, 1), (30, 8, 4096, 4, 4), (2, 16, 32768, 4, 2)])
def test_o_f32_holds_24_bits_of_the_weights(B, Sq, Sk, H, KV, hd, cap):
    from paper_2606_30634_amd import attention as T
    log(f"B {B} Sq {Sq} Sk {Sk} heads {H}/{KV} hd {hd} cap {cap}")
    q, k, v, start, end, s = _inputs(B, Sq, Sk, H, KV, hd)
    f = T.attention(q, k, v, key_start=start, key_end=end, scale=1.0, softcap=cap, keep_f32=True)
    p = np.exp(-(cap * np.tanh(s / cap) if cap else s))[:, :, None, None]
    got = f.o_f32.double().cpu().numpy()
    err = np.abs(got / (p / (1 + p)) - 1).max()
    assert err <= (26 if cap else 16) * U, err / U
