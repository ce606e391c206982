"""Dropout with the residual on the GPU against the oracle: the mask bit for bit, values within one rounding of the
product, one of the sum and one of the output, u = 2^-24 each and half a step of the type."""
import numpy as np
import pytest

from gpu_common import log
from oracle import attention as A

pytestmark = pytest.mark.gpu

HALF = {False: 2.0 ** -24, True: 2.0 ** -8}


def _matrix(r, n, c, bf16, pad, lead):
    import torch
    buf = torch.full((lead + n * (c + pad),), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    m = buf[lead:].view(n, c + pad)[:, :c]
    m.copy_(torch.from_numpy(r.normal(size=(n, c)).astype(np.float32)))
    return m, m.double().cpu().numpy()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,c", [(1, 1), (1, 7), (3, 5), (2, 8), (7, 9), (37, 515), (5, 64), (33, 40), (300, 3), (2, 2049)])
def test_dropout(n, c, bf16):
    import torch
    from paper_2606_30634_amd import dropout as D
    r = np.random.default_rng(n * 131 + c)
    for p, pad, lead, seed, offset in ((0.1, 0, 0, 1, 0), (0.5, 8, 0, 2 ** 64 - 1, 2 ** 64 - 1), (0.25, 3, 1, 123456789, 2 ** 40 + 5),
                                       (0.0, 0, 0, 5, 6), (65535 / 65536, 0, 0, 7, 8), (1e-6, 1, 0, 3, 2 ** 32)):
        log(f"rows {n} cols {c} bf16 {bf16} p {p} pad {pad} lead {lead}")
        keep, factor = A.dropout_keep(n, c, p, seed, offset)
        x, xv = _matrix(r, n, c, bf16, pad, lead)
        res, rv = _matrix(r, n, c, bf16, 2 * pad, lead)
        want = np.where(keep, xv * factor, 0.0)
        tol = 2 * HALF[False] * np.abs(want)
        got = D.dropout_backward(x, p, seed, offset)
        gv = got.double().cpu().numpy()
        assert ((gv != 0) == (keep & (xv != 0))).all()
        assert (np.abs(gv - want) <= tol + HALF[bf16] * (np.abs(want) + tol)).all()
        out = torch.full((n, c + pad), 7.0, dtype=x.dtype, device="cuda:0")
        D.dropout_add(x, res, p, seed, offset, out=out[:, :c])
        s = want + rv
        tol = tol + HALF[False] * np.abs(s)
        assert (np.abs(out[:, :c].double().cpu().numpy() - s) <= tol + HALF[bf16] * (np.abs(s) + tol)).all()
        assert bool((out[:, c:] == 7).all())
        # in place of the residual, and of x
        other = res.clone()
        D.dropout_add(x, other, p, seed, offset, out=other)
        assert torch.equal(other, out[:, :c])
        other = x.clone()
        D.dropout_add(other, res, p, seed, offset, out=other)
        assert torch.equal(other, out[:, :c])
        # what is dropped may hold anything
        x[torch.from_numpy(~keep).to("cuda:0")] = float("nan")
        assert torch.equal(D.dropout_add(x, res, p, seed, offset), out[:, :c])


@pytest.mark.parametrize("bf16", [False, True])
def test_mask_is_that_of_the_place(bf16):
    """Strides and alignment do not move the mask; offsets and seeds do; a column of counters past 2^32 elements is not
    reached here, but the counter's upper word is the oracle's."""
    import torch
    from paper_2606_30634_amd import dropout as D
    log(f"bf16 {bf16}")
    dt = torch.bfloat16 if bf16 else torch.float32
    one = torch.ones(513, 1000, dtype=dt, device="cuda:0")
    base = D.dropout_backward(one, 0.3, 11, 12)
    for pad, lead in ((8, 0), (1, 0), (0, 1), (4, 4)):
        buf = torch.ones(lead + 513 * (1000 + pad), dtype=dt, device="cuda:0")[lead:].view(513, 1000 + pad)[:, :1000]
        assert torch.equal(D.dropout_backward(buf, 0.3, 11, 12), base)
    assert abs(float((base != 0).float().mean()) - 0.7) < 4 * (0.21 / base.numel()) ** 0.5
    for seed, offset in ((11, 13), (12, 12), (11 + 2 ** 32, 12), (11, 12 + 2 ** 32)):
        same = float(((D.dropout_backward(one, 0.3, seed, offset) != 0) == (base != 0)).float().mean())
        assert abs(same - 0.58) < 0.01


def test_gradient_against_differences():
    """The mask is linear in x: a step along one direction moves the output by the gradient's product with it."""
    import torch
    from paper_2606_30634_amd import dropout as D
    r = np.random.default_rng(3)
    x, xv = _matrix(r, 40, 33, False, 0, 0)
    res, _ = _matrix(r, 40, 33, False, 0, 0)
    d, dv = _matrix(r, 40, 33, False, 0, 0)
    w, wv = _matrix(r, 40, 33, False, 0, 0)
    g = D.dropout_backward(w, 0.4, 5, 6).double()
    step = (D.dropout_add(x + d, res, 0.4, 5, 6).double() - D.dropout_add(x - d, res, 0.4, 5, 6).double()) / 2
    # three fp32 roundings of values below 16 on each side of 1320 elements
    assert abs(float((step * w.double()).sum() - (g * d.double()).sum())) < 1320 * 16 * 6 * 2.0 ** -24


def test_graph_and_stream():
    import torch
    from paper_2606_30634_amd import dropout as D
    log("graph")
    x, res = (torch.randn(777, 1031, device="cuda:0", dtype=torch.bfloat16) for _ in range(2))
    want, out = D.dropout_add(x, res, 0.1, 1, 2), torch.empty_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        D.dropout_add(x, res, 0.1, 1, 2, out=out)
    for _ in range(3):
        out.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = D.dropout_add(x, res, 0.1, 1, 2)
    s.synchronize()
    assert torch.equal(got, want)
