"""Attention over keys and values at the ends of their types' range, against float64."""
import numpy as np
import pytest
import torch

from gpu_util import gpu_available, rand, to_f64
from seq_util import Batch, sentinel

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

PAGE, D = 16, 64


@pytest.fixture(scope="module")
def ops():
    from paper_2307_04339_amd import ops as o
    return o


@pytest.fixture(scope="module")
def seq():
    from oracle import sequences
    return sequences


def _run(ops, b, x, heads, window, causal, max_q):
    y = sentinel((b.tokens, heads * D), b.dtype)
    q_start, kv_len, table = b.arrays()
    op = ops.attention(x, b.k, b.v, y, q_start, kv_len, table, heads=heads, window=window, causal=causal, max_q=max_q)
    op.run()
    torch.cuda.synchronize()
    return op, to_f64(y)


def _visible(b, s, pos, window, causal):
    """Pages of the keys that the token at pos sees."""
    hi = min(b.ctx[s], pos + 1) if causal else b.ctx[s]
    lo = max(0, pos - window + 1) if window else 0
    return set(range(lo // PAGE, (hi - 1) // PAGE + 1)) if hi > lo else set()


LOWEST = [
    # new, ctx, heads, kv_heads, window, causal, max_q, pages of each sequence whose scores are all -inf
    ([1, 1, 1], [40, 40, 0], 2, 1, 0, True, 1, [{0, 1, 2}, {0, 1}, set()]),          # all of them, some, no keys
    ([1, 1], [300, 9000], 4, 2, 0, True, 1, [set(range(19)), set(range(563))]),      # divided among tiles
    ([1], [9000], 4, 2, 0, True, 1, [set(range(400))]),                              # some tiles' keys
    ([4, 2], [40, 2], 2, 2, 18, True, 4, [{0, 1}, set()]),                           # more than one row, a window
    ([4, 2], [40, 2], 2, 2, 18, True, 4, [{1, 2}, set()]),                           # all that the window shows
    ([3], [33], 2, 2, 0, False, 4, [{0, 1, 2}]),
    ([70, 5], [70, 300], 2, 1, 0, True, None, [{0, 1}, set(range(19))]),             # early rows see nothing else
    ([40], [400], 2, 1, 33, True, None, [{22, 23}]),
    ([33], [9000], 2, 1, 0, True, None, [set(range(563))]),                          # divided among tiles
    ([33, 1], [9000, 50], 2, 1, 0, True, None, [set(range(300)), {0, 1, 2, 3}]),
    ([50, 3], [30, 2], 2, 1, 0, True, None, [{0}, set()]),                           # rows before the first key
]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", LOWEST)
def test_scores_of_minus_infinity(ops, seq, dtype, case):
    """0 / 0 where a row sees keys and all their scores are -inf; zeros where it sees none; the others' result where it
    sees others: that of a cache without the pages."""
    new, ctx, heads, kv, window, causal, max_q, low = case
    b = Batch(new, ctx, PAGE, kv, D, dtype, 300, behind=0).hide_unused()
    x, x64 = rand((b.tokens, heads * D), dtype, 301, 0.5, 2)                # positive: times -inf and summed, -inf
    without = b.table.copy()
    for s, pages in enumerate(low):
        for p in pages:
            at = int(b.table[s, p])
            n = min(PAGE, ctx[s] - p * PAGE)
            b.k[at, :, :n, 5] = float("-inf")
            without[s, p] = -1
    _, got = _run(ops, b, x, heads, window, causal, max_q)
    h = seq.HALF_STEP[dtype]
    want = seq.attention(x64, b.k64, b.v64, b.q_start, b.kv_len, without, heads, None, causal, window, None, h, 2 * h)
    for r, s, pos, _, _ in seq.tokens_of(b.q_start, b.kv_len, b.tokens, 1 << 20):
        seen = _visible(b, s, pos, window, causal)
        if not seen:
            assert np.all(got[r] == 0), r
        elif seen <= low[s]:
            assert np.all(np.isnan(got[r])), r
        else:
            assert np.all(np.abs(got[r] - want[r][0]) <= want[r][1]), r


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("max_q", [1, None])
def test_absent_pages_beside_scores_of_minus_infinity(ops, dtype, max_q):
    """Pages that are not there give a row no keys, however many there would be."""
    b = Batch([1, 1, 1], [200, 200, 200], PAGE, 1, D, dtype, 310, behind=0, beyond=0)
    b.table[0, :] = -1                                  # nothing is there
    b.table[1, :-1] = -1                                # one page is, all -inf
    x, _ = rand((3, 2 * D), dtype, 311, 0.5, 2)
    b.k[int(b.table[1, -1]), :, :, 0] = float("-inf")
    b.k[int(b.table[2, 3]), :, :, 0] = float("-inf")
    _, got = _run(ops, b, x, 2, 0, True, max_q)
    assert np.all(got[0] == 0) and np.all(np.isnan(got[1])) and np.all(np.isfinite(got[2])) and np.all(got[2] != 0)
