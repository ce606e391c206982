"""Pins of the oracle's attention over key ranges, key ranges and dropout: small cases by hand, the gradient against
central differences in float64, and Philox4x32-10 against the published vectors of its paper's library."""
import numpy as np
import pytest

from oracle import attention as A


def test_ranges_by_hand():
    ids = np.array([[5, 5, 5, 7, 7, -1, 5, 5], [-3, -3, 0, 1, 1, 1, 1, -1]])
    start, end = A.key_ranges(ids)
    assert start.tolist() == [[0, 0, 0, 3, 3, 0, 6, 6], [0, 0, 2, 3, 3, 3, 3, 0]]
    assert end.tolist() == [[1, 2, 3, 4, 5, 0, 7, 8], [0, 0, 3, 4, 5, 6, 7, 0]]
    flags = np.array([[1, 1, 0, 0, 1, 1, 1, 1], [1, 1, 1, 1, 1, 0, 1, 1]])
    start, end = A.key_ranges(ids, flags)
    assert end.tolist() == [[2, 2, 3, 4, 5, 0, 8, 8], [0, 0, 3, 5, 5, 6, 7, 0]]


def test_attention_by_hand():
    q, k = np.zeros((1, 2, 1, 2)), np.zeros((1, 3, 1, 2))
    v = np.arange(6.0).reshape(1, 3, 1, 2)
    o, lse = A.attention(q, k, v, np.array([[0, 2]]), np.array([[2, 2]]))
    assert o[0, 0, 0].tolist() == [1.0, 2.0] and not o[0, 1].any()
    assert np.isclose(lse[0, 0, 0], np.log(2)) and lse[0, 0, 1] == -np.inf
    # a distance of d lowers a score by slope d; the cap bends x to cap tanh(x / cap)
    q[0, 0, 0], k[0, :, 0, 0] = (3.0, 0.0), (1.0, 2.0, 3.0)
    _, lse = A.attention(q, k, v, np.array([[0, 0]]), np.array([[3, 0]]), q_start=[2], scale=1.0, cap=4.0, slopes=np.array([0.5]))
    assert np.isclose(lse[0, 0, 0], np.log(sum(np.exp(4 * np.tanh(3 * x / 4) - 0.5 * d) for x, d in ((1, 2), (2, 1), (3, 0)))))


@pytest.mark.parametrize("cap,bias", [(0.0, False), (2.0, True)])
def test_gradient_against_differences(cap, bias):
    r = np.random.default_rng(5)
    B, Sq, Sk, H, KV, hd = 2, 4, 5, 4, 2, 3
    q, k, v = r.normal(size=(B, Sq, H, hd)), r.normal(size=(B, Sk, KV, hd)), r.normal(size=(B, Sk, KV, hd))
    start = np.array([[0, 0, 2, 3], [1, 0, 0, 0]])
    end = np.array([[1, 4, 5, 3], [5, 2, 3, 5]])
    kw = dict(q_start=[1, 3], scale=0.7, cap=cap, slopes=r.uniform(0.1, 0.5, size=H) if bias else None)
    do = r.normal(size=q.shape)
    got = A.attention_bwd(q, k, v, do, start, end, **kw)
    for x, g in zip((q, k, v), got):
        for i in np.ndindex(x.shape):
            keep, eps = x[i], 1e-6
            x[i] = keep + eps
            hi = (A.attention(q, k, v, start, end, **kw)[0] * do).sum()
            x[i] = keep - eps
            lo = (A.attention(q, k, v, start, end, **kw)[0] * do).sum()
            x[i] = keep
            assert abs((hi - lo) / (2 * eps) - g[i]) < 1e-8


def test_philox_vectors():
    """The known-answer vectors published with the generator."""
    hexes = lambda w: " ".join(f"{x:08x}" for x in w)  # noqa: E731
    ones = 0xFFFFFFFF
    assert hexes(A.philox((0, 0, 0, 0), (0, 0))) == "6627e8d5 e169c58d bc57ac4c 9b00dbd8"
    assert hexes(A.philox((ones,) * 4, (ones,) * 2)) == "408f276d 41c83b0e a20bc7c6 6d5451fd"
    assert hexes(A.philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0))) == \
        "d16cfe09 94fdcceb 5001e420 24126ea1"


def test_dropout_keeps_its_share():
    keep, factor = A.dropout_keep(50, 41, 0.25, 7, 3)
    assert factor == 4 / 3 and abs(keep.mean() - 0.75) < 4 * np.sqrt(0.25 * 0.75 / keep.size)
    assert A.dropout_keep(3, 5, 0.0, 1, 2)[0].all()
