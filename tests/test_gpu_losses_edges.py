"""Log-probability and loss operators at edges of their own: inputs taken in chunks, workspaces of exactly the size
asked for, values at the ends of the types.  Against the oracle in float64; bounds count roundings, u = 2^-24, as the
operators' other tests do."""
import numpy as np
import pytest

from gpu_common import log
from oracle import losses as L
from test_gpu_losses import U, _err, _f32, _head_tol, _i32, _matrix, _np

pytestmark = pytest.mark.gpu


def _guarded(need, guard=65536):
    """A uint8 workspace of `need` bytes with a pattern behind it, and the check that the pattern is whole."""
    import torch
    buf = torch.full((need + guard,), 0xA5, dtype=torch.uint8, device="cuda:0")
    return buf[:need], lambda: bool((buf[need:] == 0xA5).all())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,v,d", [(712, 16384, 33), (600, 20000, 33), (129, 128256, 33), (99, 128256, 5), (1300, 8193, 1)])
def test_head_of_unaligned_rows_in_chunks(n, v, d, bf16):
    """Rows that are not whole 16 bytes go through fp32 logits, 32 MiB of them at a time: several chunks, the last of
    them smaller and split further than the others.  Nothing is written behind the workspace."""
    from paper_2606_30634_amd import binding as B
    from paper_2606_30634_amd import losses
    r = np.random.default_rng(n + v)
    mx, xv = _matrix(r.normal(size=(n, d)), bf16, pad=2)
    mw, wv = _matrix(r.normal(size=(v, d)) * (2 / np.sqrt(d)), bf16, lead=1)
    t = r.integers(0, v, size=n)
    t[n // 3], t[n - 2] = -1, v
    rows = np.unique(np.r_[0:n:37, n // 3, n // 2, n - 34:n])  # the oracle's share of them
    log(f"rows {n} vocab {v} d {d} bf16 {bf16}")
    need = B.head_logprob_workspace_bytes(n, v, d, bf16)
    ws, whole = _guarded(need)
    got = losses.head_logprob(mx, mw, _i32(t), inv_temperature=1.5, workspace=ws)
    assert whole()
    ref = L.token_logprob(xv[rows] @ wv.T, t[rows], 1.5)
    e = _head_tol(d, xv[rows], wv, 1.5)
    lp, ent, st = (_np(a)[rows] for a in got)
    assert (np.abs(lp - ref[0]) <= 2 * e + _err(v, ref[0])).all()
    assert (np.abs(st[:, 0] - ref[2][:, 0]) <= e / 1.5).all()
    assert (np.abs(st[:, 1] - ref[2][:, 1]) <= 2 * e + _err(v, 0.0)).all()
    assert (np.abs(ent - ref[1]) <= (2 * e + 2 * _err(v, 0.0)) * 2 * (np.abs(ref[2][:, 1]) + 1 + np.log(v))).all()
    gone = (t < 0) | (t >= v)
    assert gone.sum() == 2 and not _np(got.logp)[gone].any() and _np(got.logp)[~gone].all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,v,d", [(1, 300, 64), (24, 30000, 64), (45, 10902, 2144), (300, 777, 1000), (333, 32001, 512),
                                   (16400, 264, 64), (700, 9001, 2996)])
def test_head_workspace_is_enough(n, v, d, bf16):
    """Every way the fused product lays out its workspace: row tiles, packed rows, more rows than one product takes."""
    import torch
    from paper_2606_30634_amd import binding as B
    from paper_2606_30634_amd import losses
    g = torch.Generator(device="cuda:0").manual_seed(n)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = torch.randn(n, d, generator=g, device="cuda:0").to(dt)
    w = (torch.randn(v, d, generator=g, device="cuda:0") / d ** 0.5).to(dt)
    t = torch.randint(-v // 4, v, (n,), generator=g, device="cuda:0", dtype=torch.int32)
    log(f"rows {n} vocab {v} d {d} bf16 {bf16}")
    ws, whole = _guarded(B.head_logprob_workspace_bytes(n, v, d, bf16))
    got = losses.head_logprob(x, w, t, workspace=ws)
    assert whole()
    other = losses.head_logprob(x, w, t)
    assert all(torch.equal(a, b) for a, b in zip(got, other))


def test_other_workspaces_are_enough():
    """Rows of logits in parts, and the losses above and below the sizes that one block takes."""
    import torch
    from paper_2606_30634_amd import binding as B
    from paper_2606_30634_amd import losses
    for n, v in ((1, 16384), (5, 40001), (34, 128256), (256, 16390), (513, 20000)):
        log(f"rows {n} vocab {v}")
        x = torch.randn(n, v, device="cuda:0")
        t = torch.randint(-2, v, (n,), device="cuda:0", dtype=torch.int32)
        ws, whole = _guarded(B.token_logprob_workspace_bytes(n, v))
        losses.token_logprob(x, t, workspace=ws)
        assert whole()
    for b, s in ((1, 1), (8, 1024), (9, 1024), (1026, 3), (2, 40001), (600, 2048), (70000, 2)):
        log(f"sequences {b} length {s}")
        lp = -torch.rand(b, s, device="cuda:0")
        on = torch.rand(b, s, device="cuda:0") < 0.7
        ws, whole = _guarded(B.policy_loss_workspace_bytes(b, s))
        losses.policy_loss(lp, lp + 0.1, lp[:, 0].contiguous(), on, workspace=ws)
        assert whole()
        if b % 2 == 0:
            ws, whole = _guarded(B.preference_loss_workspace_bytes(b // 2, s))
            losses.preference_loss(lp, on, workspace=ws)
            assert whole()
