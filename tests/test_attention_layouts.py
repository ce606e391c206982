"""Where the three gradients of attention may lie: layouts in which two of them share an element are refused, layouts that only
interleave are not.  Through the C ABI, without a device (what is accepted is stopped by the check of its workspace, the
last one)."""
import pytest

from paper_2606_30634_amd import binding as B

P, Q = 1 << 40, 1 << 44  # aligned addresses that are never read
BASE = dict(batch=2, queries=5, keys=5, heads=4, kv=2, hd=64)


def _message(at, strides, **kw):
    """at, strides: of dq, dk and dv in bf16, elements"""
    d = dict(BASE, **kw)
    hd = d["hd"]
    q, k = d["heads"] * hd, d["kv"] * hd
    sq, sk = B._STRIDES(d["queries"] * q, q, hd), B._STRIDES(d["keys"] * k, k, hd)
    p = B.AttentionParams(d["batch"], d["queries"], d["keys"], d["heads"], d["kv"], hd, 1, sq, sk, sk, None, None, None, None, 0.125, 0.0)
    g = B.AttentionGrads(sq, sq, *(B._STRIDES(*s) for s in strides), *(Q + 2 * a for a in at), 0)
    with pytest.raises(B.StageError) as e:
        B.attention_backward(p, P, P, P, P, P, P, g, None, 0, None)
    assert e.value.code == B.STAGE_EINVAL
    return B.last_error()


def _rows_first(W):
    """[S, B, W]: a batch stride of W, a row stride of B W"""
    return [(W, 2 * W, 64)] * 3


@pytest.mark.parametrize("name,at,strides", [
    ("dv of one sequence on dk of the next", (0, 256, 256 + 512), _rows_first(512)),
    ("the same, the other way round", (0, 256 + 512, 256), _rows_first(512)),
    ("dk half a row on", (0, 256, 512 + 64), _rows_first(512)),
    ("dq of the next sequence on dv", (512, 256, 384), _rows_first(448))])
def test_rows_that_meet_over_the_batch(name, at, strides):
    assert "overlap" in _message(at, strides), name


@pytest.mark.parametrize("name,at,strides", [
    ("packed rows [B, S, W]", (0, 256, 384), [(2560, 512, 64)] * 3),
    ("packed rows [S, B, W]", (0, 256, 384), _rows_first(512)),
    ("apart", (0, 1 << 20, 1 << 21), [(1280, 256, 64), (640, 128, 64), (640, 128, 64)])])
def test_rows_that_do_not(name, at, strides):
    assert "workspace" in _message(at, strides), name
