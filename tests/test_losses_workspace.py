"""Sizes that the workspace calls give against what the operators lay out in them: arithmetic alone, no device."""
import pytest

from paper_2606_30634_amd import binding as B

HELD = 32 << 20  # bytes of fp32 logits that a head of unaligned rows holds at once


def _up(n, to=256):
    return (n + to - 1) // to * to


def _chunk(rows, vocab):
    r = min(HELD // (4 * vocab), 1 << 20)
    return max(1, min(rows, r // 128 * 128 if r > 128 else r))


@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("vocab", [1, 2, 777, 8191, 16384, 17000, 20000, 24577, 32001, 49153, 70001, 128256, 524288, 1 << 24])
def test_head_workspace_covers_every_chunk(vocab, bf16):
    """A head of unaligned rows (d = 33) takes them a chunk at a time: the chunk's logits, then the parts of its rows,
    whose number grows as the rows become fewer, so that the last chunk's can be the larger ones."""
    for rows in sorted({*range(1, 1200, 7), 64, 65, 128, 129, 512, 600, 640, 712, 2000, 16384, 16385, 70000, 1 << 30}):
        have = B.head_logprob_workspace_bytes(rows, vocab, 33, bf16)
        r = _chunk(rows, vocab)
        for n in {r, (rows - 1) % r + 1}:
            need = _up(r * vocab * 4) + B.token_logprob_workspace_bytes(n, vocab)
            assert have >= need, (rows, n, have, need)


@pytest.mark.parametrize("vocab", [1, 2, 3])
def test_head_chunk_fits_a_grid(vocab):
    """Chunks of a head of a token or two: their tiles of 64 rows within the 65536 of a grid's second dimension."""
    assert B.head_logprob_workspace_bytes(9_000_001, vocab, 1, 1) <= _up(65536 * 64 * vocab * 4)
