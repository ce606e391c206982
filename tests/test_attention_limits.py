"""Calls whose launches would pass what a launch takes are refused before anything is launched, and calls just within it
are not: through the C ABI, without a device (the accepted ones are stopped by the check of their workspace, the last one)."""
import pytest

from paper_2606_30634_amd import binding as B

P, Q, R = 1 << 60, 1 << 61, 3 << 60  # aligned addresses, far from each other, that are never read


def _params(batch, queries, keys, heads, kv, hd, bf16):
    s = lambda n, h: B._STRIDES(n * h * hd, h * hd, hd)  # noqa: E731
    return B.AttentionParams(batch, queries, keys, heads, kv, hd, int(bf16), s(queries, heads), s(keys, kv), s(keys, kv), None, None,
                             None, None, 0.125, 0.0)


def _message(fn, *args):
    with pytest.raises(B.StageError) as e:
        fn(*args)
    assert e.value.code == B.STAGE_EINVAL
    return B.last_error()


def _backward(p):
    q, k = p.queries * p.heads * p.head_dim, p.keys * p.kv_heads * p.head_dim
    hd = p.head_dim
    sq, sk = B._STRIDES(q, p.heads * hd, hd), B._STRIDES(k, p.kv_heads * hd, hd)
    g = B.AttentionGrads(sq, sq, sq, sk, sk, Q, R, R + (1 << 58), 0)
    return _message(B.attention_backward, p, P, P + (1 << 58), P + (1 << 59), P, P, P, g, None, 0, None)


@pytest.mark.parametrize("batch,queries,heads,hd,bf16,ok", [
    (4096, 1024, 32, 128, True, False),    # 2^34 elements of q: 2^24 blocks of statistics
    (4064, 1024, 32, 128, True, True),
    (4096, 1024, 64, 64, True, False),
    (4060, 1024, 64, 64, True, True),
    (8192, 2048, 32, 32, True, False),
    (1 << 18, 1, 32, 128, True, True),
    (256, 32768, 64, 32, False, False),    # 2^24 blocks of 32 queries, and those of the keys
    (255, 32768, 32, 32, False, True)])
def test_the_backward_fits_a_launch(batch, queries, heads, hd, bf16, ok):
    m = _backward(_params(batch, queries, queries, heads, 1, hd, bf16))
    assert ("workspace" in m) == ok and ("too large" in m) == (not ok), m


@pytest.mark.parametrize("batch,queries,heads,hd,bf16,ok", [
    (512, 32768, 32, 64, False, False), (511, 32768, 32, 64, False, True), (8192, 33, 1024, 32, False, False),
    (512, 32768, 32, 64, True, True)])
def test_the_forward_fits_a_launch(batch, queries, heads, hd, bf16, ok):
    p = _params(batch, queries, 16, heads, 1, hd, bf16)
    # (what is not split needs no workspace: an output over an input is what stops the call that fits)
    m = _message(B.attention_forward, p, P, P + (1 << 58), P + (1 << 59), Q, None, R, None, 0, None) if not ok else \
        _message(B.attention_forward, p, P, P + (1 << 58), P + (1 << 59), P, None, R, None, 0, None)
    assert ("overlap" in m) == ok and ("too large" in m) == (not ok), m
