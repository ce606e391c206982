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


def _slices(heads, S):
    """[B, heads, S, 64] transposed"""
    return [(heads * S * 64, 64, S * 64)] * 3


@pytest.mark.parametrize("name,at,strides,kw", [
    ("packed single tokens", (0, 256, 384), [(512, 0, 64)] * 3, dict(queries=1, keys=1)),
    ("one query on packed keys", (0, 1 << 20, (1 << 20) + 128), [(256, 0, 64), (1280, 256, 64), (1280, 256, 64)], dict(queries=1)),
    ("dk and dv head by head", (0, 1 << 20, (1 << 20) + 64), [(1280, 256, 64), (1280, 256, 128), (1280, 256, 128)], {}),
    ("all three head by head", (0, 64, 128), [(3840, 768, 192)] * 3, dict(kv=4)),
    ("slices of [B, heads, S, hd]", (0, 1280, 1920), _slices(8, 5), {}),
    ("dk over even and dv over odd rows", (0, 1 << 20, (1 << 20) + 128), [(1280, 256, 64), (1280, 256, 64), (1280, 256, 64)], {}),
    ("one sequence of packed rows", (0, 256, 384), [(0, 512, 64)] * 3, dict(batch=1))])
def test_rows_that_interleave(name, at, strides, kw):
    assert "workspace" in _message(at, strides, **kw), name


@pytest.mark.parametrize("name,at,strides,kw", [
    ("packed single tokens of the next sequence", (0, 256, 256 + 512), [(512, 0, 64)] * 3, dict(queries=1, keys=1)),
    ("dv on dk, head by head", (0, 1 << 20, (1 << 20) + 128), [(1280, 256, 64), (1280, 256, 128), (1280, 256, 128)], {}),
    ("half a head", (0, 1 << 20, (1 << 20) + 32), [(1280, 256, 64), (1280, 256, 128), (1280, 256, 128)], {}),
    ("slices that meet", (0, 1280 - 64, 1920), _slices(8, 5), {}),
    ("dk of the next sequence", (0, 1280, 1280 + 2240), _slices(7, 5), {}),
    ("other strides", (0, 128, 256), [(2560, 512, 64), (1280, 256, 64), (2560, 512, 64)], {})])
def test_interleaved_rows_that_meet(name, at, strides, kw):
    assert "overlap" in _message(at, strides, **kw), name


def test_against_every_element():
    """Random layouts: what is accepted shares no element."""
    import itertools
    import random
    rng = random.Random(3)
    accepted = 0
    for _ in range(4000):
        kw = dict(batch=rng.choice([1, 2, 3]), queries=rng.choice([1, 2, 3]), heads=rng.choice([1, 2, 4]), kv=1, hd=32)
        kw.update(keys=rng.choice([kw["queries"], 2]), kv=rng.choice([k for k in (1, 2, 4) if kw["heads"] % k == 0]))
        common = [rng.choice([0, 32, 64, 96, 128, 192, 256, 384, 512, 768]) for _ in range(3)]
        strides = [tuple(c if rng.random() < 0.85 else rng.choice([32, 64, 128, 256]) for c in common) for _ in range(3)]
        at = [32 * rng.randrange(0, 24) for _ in range(3)]
        m = _message(at, strides, **kw)
        if "workspace" not in m:
            assert "overlap" in m
            continue
        accepted += 1
        seen = set()
        for a, s, n in zip(at, strides, ((kw["queries"], kw["heads"]), (kw["keys"], kw["kv"]), (kw["keys"], kw["kv"]))):
            for b, i, h in itertools.product(range(kw["batch"]), range(n[0]), range(n[1])):
                e = a + b * s[0] + i * s[1] + h * s[2]
                rows = set(range(e, e + 32))
                assert not rows & seen, (at, strides, kw)
                seen |= rows
    assert accepted > 50
