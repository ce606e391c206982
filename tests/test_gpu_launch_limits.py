"""Documented sizes that pass the 2^32 threads of one launch."""
import pytest

from gpu_common import log
from oracle import attention as A

pytestmark = pytest.mark.gpu


def test_dropout_past_one_launch():
    """2^35 elements and more: the mask of their places on both sides of where the second launch starts."""
    import torch
    from paper_2606_30634_amd import dropout as D
    rows, cols, seed, offset = (1 << 15) + 3, 1 << 20, 77, 5
    log(f"rows {rows} cols {cols}")
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 64 GiB of free device memory")
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda:0")
    D.dropout_backward(x, 0.5, seed, offset, out=x)
    flat = x.view(-1)
    n, second = rows * cols, 256 * 8 * ((1 << 24) - 1)
    for at in (0, second - 512, second, 1 << 35, n - 512):
        want = []
        for g in range(at // 8, at // 8 + 64):
            for w in A.philox((g & 0xFFFFFFFF, g >> 32, offset, 0), (seed, 0)):
                want += [w & 0xFFFF, w >> 16]
        want = (torch.tensor(want) >= 32768).float() * 2
        assert torch.equal(flat[at:at + 512].float().cpu(), want), at
    kept = torch.stack([(flat[a:a + (1 << 30)] != 0).float().mean() for a in (0, second - (1 << 29), n - (1 << 30))])
    assert bool(((kept - 0.5).abs() < 2.0 ** -12).all())  # 16 standard deviations of the mean of 2^30


@pytest.mark.parametrize("length,prefix", [(1, False), (2, True)])
def test_key_ranges_past_one_launch(length, prefix):
    """2^24 rows, as many as are allowed."""
    import torch
    from paper_2606_30634_amd import attention as T
    rows = 1 << 24
    log(f"rows {rows} length {length} prefix {prefix}")
    g = torch.Generator(device="cuda:0").manual_seed(length)
    ids = torch.randint(-1, 2, (rows, length), generator=g, device="cuda:0", dtype=torch.int32)
    flags = torch.randint(0, 2, (rows, length), generator=g, device="cuda:0", dtype=torch.uint8) if prefix else None
    start, end = T.key_ranges(ids, prefix=flags)
    live = ids >= 0
    ws, we = torch.zeros_like(ids), live.int()
    if length == 2:
        same = live[:, 1] & (ids[:, 0] == ids[:, 1])
        ws[:, 1] = torch.where(live[:, 1] & ~same, 1, 0)
        we[:, 1] = torch.where(live[:, 1], 2, 0)
        we[:, 0] = torch.where(same & (flags != 0).all(1), 2, we[:, 0])
    assert torch.equal(start, ws) and torch.equal(end, we)
