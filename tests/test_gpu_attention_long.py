"""Attention over key ranges at lengths where its work is shared out: more key blocks than are ordered by their queries,
many shares of few key or query blocks; and key ranges of documents over many blocks.  Bounds as in test_gpu_attention.py."""
import numpy as np
import pytest

from gpu_common import log
from test_gpu_attention import _case, _check_backward, _check_forward, _fast_ranges, _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16,hd", [(True, 32), (True, 64), (True, 128), (False, 64)])
@pytest.mark.parametrize("B,Sq,Sk,H,KV", [(1, 260, 33000, 2, 1), (2, 70, 32900, 1, 1), (1, 4100, 250, 4, 1), (1, 130, 16400, 2, 1)])
def test_long(B, Sq, Sk, H, KV, bf16, hd):
    log(f"B {B} Sq {Sq} Sk {Sk} heads {H}/{KV} hd {hd} bf16 {bf16}")
    x, how, rng, ref = _case(Sq + Sk, B, Sq, Sk, H, KV, hd, bf16, "random", cap=20.0, bias=hd == 64, qstd=2.0)
    f = _check_forward(x, how, rng, ref, bf16, bf16)
    _check_backward(x, how, rng, ref, bf16, f)


@pytest.mark.parametrize("rows,length,docs", [(1, 131077, 1), (3, 70001, 2), (2, 131072, 40)])
@pytest.mark.parametrize("prefix", [0, 0.5, 1])
def test_long_documents(rows, length, docs, prefix):
    import torch
    from paper_2606_30634_amd import attention as T
    log(f"rows {rows} length {length} documents {docs} prefix {prefix}")
    r = np.random.default_rng(length + docs)
    cut = np.sort(r.integers(0, length, size=(rows, docs - 1)), 1)
    ids = (np.arange(length)[None, :, None] >= cut[:, None, :]).sum(2).astype(np.int32) - (docs > 2)
    flags = None
    if prefix:
        flags = np.ones((rows, length), np.uint8)
        for b in range(rows):
            for lo, hi in zip([0, *cut[b]], [*cut[b], length]):
                flags[b, lo + int(prefix * (hi - lo)):hi] = 0
    start, end = T.key_ranges(_i32(ids), prefix=None if flags is None else torch.from_numpy(flags).to("cuda:0"))
    ws, we = _fast_ranges(ids, flags)
    np.testing.assert_array_equal(start.cpu().numpy(), ws)
    np.testing.assert_array_equal(end.cpu().numpy(), we)
