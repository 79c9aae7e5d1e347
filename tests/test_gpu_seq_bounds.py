"""Starts, lengths and pages of any value: every buffer lies between guards that must not change, rows that belong to
no sequence and places that belong to no token are left as they were, and the others are compared with float64, whose
oracle clamps the same arrays by itself."""
import numpy as np
import pytest
import torch

from gpu_util import TORCH, bits, gpu_available, rand, to_f64

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

GUARD = 1 << 14
BIG, LOW = 2 ** 31 - 1, -2 ** 31


@pytest.fixture(scope="module")
def ops():
    from paper_2307_04339_amd import ops as o
    return o


@pytest.fixture(scope="module")
def seq():
    from oracle import sequences
    return sequences


class Guarded:
    """A contiguous tensor between two guards (NaN for what is read, so that a value from there shows)."""

    def __init__(self, like, dtype, fill):
        n = like.numel()
        self.buf = torch.full((n + 2 * GUARD,), fill, dtype=TORCH[dtype], device="cuda")
        self.t = self.buf[GUARD:GUARD + n].view(like.shape)
        self.t.copy_(like)
        self.before = (bits(self.buf[:GUARD]), bits(self.buf[GUARD + n:]))

    def untouched(self):
        n = self.t.numel()
        return (bits(self.buf[:GUARD]), bits(self.buf[GUARD + n:])) == self.before


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


PAGE, PAGES, MAX_PAGES, TOKENS, D = 16, 20, 5, 11, 64
ARRAYS = [
    # starts, lengths, values of some entries of the page table
    ([0, 1, 2, 3, 4], [BIG, LOW, -1, 70], {}),
    ([0, 4, 4, 7, 9], [70, 80, 3, 1], {}),                        # an empty sequence, more tokens than keys
    ([0, 2, 50, 60, BIG], [64, 80, 64, 64], {}),                  # starts behind the last row
    ([0, 0, 0, 0, 0], [64, 64, 64, 64], {}),                      # no tokens
    ([3, 5, 6, 8, 11], [80, 79, 17, 16], {}),                     # rows before the first sequence
    ([LOW, 2, 3, 7, 9], [20, 30, 40, 50], {}),
    ([0, 3, 6, 8, 10], [64] * 4, {(0, 0): BIG, (1, 0): LOW, (1, 3): -1, (2, 3): PAGES, (3, 1): 10 ** 6}),
    ([0, 3, 6, 8, 10], [80] * 4, {(s, p): -1 for s in range(4) for p in range(MAX_PAGES)}),
    ([BIG, LOW, 3, 1, BIG], [64] * 4, {}),                        # in no order: guards only
    ([-5, 2, 1, 9, 2], [10] * 4, {}),
    ([9, 7, 5, 3, 1], [BIG] * 4, {(2, 2): BIG}),
]


def _table(changes):
    t = np.random.default_rng(500).permutation(PAGES)[:4 * MAX_PAGES].reshape(4, MAX_PAGES).astype(np.int32)
    for at, v in changes.items():
        t[at] = v
    return t


def _in_order(starts):
    return all(b >= a for a, b in zip(starts, starts[1:]))


@pytest.mark.parametrize("window", [0, 9])
@pytest.mark.parametrize("heads,kv,max_q", [(2, 1, 1), (2, 2, 4), (2, 1, None), (32, 1, 2), (8, 2, 5)])
@pytest.mark.parametrize("arrays", ARRAYS)
def test_attention_stays_inside(ops, seq, arrays, heads, kv, max_q, window):
    starts, lens, changes = arrays
    table = _table(changes)
    nan = float("nan")
    x, x64 = rand((TOKENS, heads * D), "f16", 501, -2, 2)
    (k, k64), (v, v64) = (rand((PAGES, kv, PAGE, D), "f16", 502 + i, -1.5, 1.5) for i in range(2))
    gx, gk, gv = Guarded(x, "f16", nan), Guarded(k, "f16", nan), Guarded(v, "f16", nan)
    gy = Guarded(torch.full((TOKENS, heads * D), -77.0), "f16", -77.0)
    op = ops.attention(gx.t, gk.t, gv.t, gy.t, _ints(starts), _ints(lens), _ints(table), heads=heads, window=window, max_q=max_q)
    for block in (256, 64):
        gy.t.fill_(-77.0)
        op.launch(0, op.T, op.T, block)
        torch.cuda.synchronize()
        assert all(g.untouched() for g in (gx, gk, gv, gy))
        got = to_f64(gy.t)
        assert np.all(np.isfinite(got))
        if not _in_order(starts):
            continue
        h = seq.HALF_STEP["f16"]
        want = seq.attention(x64, k64, v64, starts, lens, table, heads, window=window, max_q=max_q, half_step=h, p_step=2 * h)
        for r in range(TOKENS):
            if r in want:
                assert np.all(np.abs(got[r] - want[r][0]) <= want[r][1]), r
            else:
                assert np.all(got[r] == -77.0), r


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("arrays", ARRAYS)
def test_rotary_stays_inside(ops, seq, arrays, inter, dtype):
    starts, lens, changes = arrays
    table = _table(changes)
    heads, kv = 3, 2
    x, x64 = rand((TOKENS, (heads + 2 * kv) * D), dtype, 510, -2, 2)
    gx = Guarded(x, dtype, float("nan"))
    gy = Guarded(torch.full((TOKENS, heads * D), -77.0), dtype, -77.0)
    gk, gv = (Guarded(torch.full((PAGES, kv, PAGE, D), -77.0), dtype, -77.0) for _ in range(2))
    freq = ops.rotary_freqs(D)
    ops.rotary(gx.t, gy.t, freq.cuda(), _ints(starts), _ints(lens), heads=heads, head_dim=D, kv_heads=kv, k_cache=gk.t, v_cache=gv.t,
               page_table=_ints(table), interleaved=inter).run()
    torch.cuda.synchronize()
    assert all(g.untouched() for g in (gx, gy, gk, gv))
    y, k, v = to_f64(gy.t), to_f64(gk.t), to_f64(gv.t)
    assert np.all(np.isfinite(y)) and np.all(np.isfinite(k)) and np.all(np.isfinite(v))
    if not _in_order(starts):
        return
    q, at = seq.rotary(x64, freq.numpy(), starts, lens, heads, kv, D, table, PAGE, PAGES, inter)
    h = seq.HALF_STEP[dtype]
    for r in range(TOKENS):
        if r in q:
            assert np.all(np.abs(y[r] - q[r][0]) <= q[r][1] * (1 + h) + h * np.abs(q[r][0]) + 2.0 ** -25), r
        else:
            assert np.all(y[r] == -77.0), r
    stored = np.zeros((PAGES, PAGE), dtype=bool)
    for (p, s), (kk, ke, vv) in at.items():
        stored[p, s] = True
        assert np.all(np.abs(k[p, :, s] - kk) <= ke * (1 + h) + h * np.abs(kk) + 2.0 ** -25), (p, s)
        assert np.array_equal(v[p, :, s], vv)
    for c in (k, v):
        assert np.all(c.transpose(0, 2, 1, 3)[~stored] == -77.0)


@pytest.mark.parametrize("heads,kv,d", [(32, 1, 64), (8, 2, 128), (20, 4, 80)])
def test_rows_behind_max_q_are_left_by_the_kernel_for_many(ops, seq, heads, kv, d):
    """Sequences of more new tokens than max_q: their first max_q rows are right, the others as they were."""
    new, ctx, max_q = [9, 1, 5, 40], [30, 20, 200, 41], 5
    rng = np.random.default_rng(520)
    need = [-(-c // PAGE) for c in ctx]
    order = rng.permutation(sum(need))
    table = np.full((4, max(need)), -1, dtype=np.int32)
    for s, n in enumerate(need):
        table[s, :n] = order[sum(need[:s]):sum(need[:s]) + n]
    starts = np.concatenate([[0], np.cumsum(new)])
    x, x64 = rand((sum(new) + 1, heads * d), "bf16", 521, -2, 2)
    (k, k64), (v, v64) = (rand((sum(need), kv, PAGE, d), "bf16", 522 + i, -1.5, 1.5) for i in range(2))
    gy = Guarded(torch.full((sum(new) + 1, heads * d), -77.0), "bf16", -77.0)
    assert max_q * heads // kv > 16
    ops.attention(x, k, v, gy.t, _ints(starts), _ints(ctx), _ints(table), heads=heads, max_q=max_q).run()
    torch.cuda.synchronize()
    got, h = to_f64(gy.t), seq.HALF_STEP["bf16"]
    want = seq.attention(x64, k64, v64, starts, ctx, table, heads, max_q=max_q, half_step=h, p_step=2 * h)
    assert len(want) == 5 + 1 + 5 + 5 and gy.untouched()
    for r in range(len(got)):
        if r in want:
            assert np.all(np.abs(got[r] - want[r][0]) <= want[r][1]), r
        else:
            assert np.all(got[r] == -77.0), r
