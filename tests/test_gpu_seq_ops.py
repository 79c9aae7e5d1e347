"""GPU parity of the operators over packed token rows (block norms, rotary positions with the append to the
paged cache, attention over it) against float64, each output within the bound of its own arithmetic; bitwise
invariance across shard plans and blocks; places that must not be read or written; replays of a captured graph
with other lengths; the operators one after another, alone and as tasks of the coordinator."""
import ctypes

import numpy as np
import pytest
import torch

from gpu_util import bits, f32_dev, gpu_available, rand, to_f64
from seq_util import Batch, elastic_bitwise, sentinel, strided

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

DTYPES = ["f32", "f16", "bf16"]


@pytest.fixture(scope="module")
def ops():
    from paper_2307_04339_amd import ops as o
    return o


@pytest.fixture(scope="module")
def seq():
    from oracle import sequences
    return sequences


def _inside(got, want, bound, what):
    assert np.all(np.isfinite(got)), what
    off = np.abs(got - want) - bound
    assert np.max(off) <= 0, (what, float(np.max(off)), float(np.max(np.abs(got - want) / bound)))


# ------------------------------------------------------------------ block norm
NORM_CASES = [
    # rows, n, norm, post, gate, residual, y, z, strided, scale
    (1, 1, "rms", True, "none", True, True, True, 0, 1.0),
    (1, 768, "rms", True, "none", True, True, True, 0, 1.0),
    (5, 768, "layer", True, "silu", True, True, True, 8, 0.5),
    (130, 64, "rms", False, "channel", True, True, True, 0, -0.25),
    (33, 7, "layer", True, "sigmoid", True, True, True, 3, 1.0),
    (9, 500, "rms", True, "rows", False, True, False, 0, 2.0),
    (7, 1021, "layer", False, "none", True, False, True, 1, 0.22),
    (6, 2050, "layer", True, "silu", True, True, True, 0, 0.5),
    (300, 4096, "rms", True, "channel", True, True, True, 0, 0.25),
    (3, 5000, "rms", False, "none", True, True, True, 8, 1.0),
    (4, 8191, "rms", True, "sigmoid", True, True, True, 5, 1.0),
    (3, 16384, "rms", True, "none", True, True, True, 0, 1.0),
    (2, 20011, "layer", True, "silu", True, True, True, 2, 0.7),
    (1030, 256, "rms", False, "none", False, False, True, 0, 1.0),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", NORM_CASES)
def test_block_norm(ops, seq, orc, dtype, case):
    m, n, norm, has_post, gate, has_res, has_y, has_z, extra, scale = case
    x, x64 = rand((m, n), dtype, 1, -2, 3)
    r, r64 = rand((m, n), dtype, 2) if has_res else (None, None)
    rng = np.random.default_rng(3)
    vec = lambda lo, hi: rng.uniform(lo, hi, n).astype(np.float32).astype(np.float64)  # noqa: E731
    post = vec(0.5, 1.5) if has_post else None
    post_b = vec(-0.5, 0.5) if has_post and norm == "layer" else None
    pre = vec(-1.5, 1.5) if has_z else None
    pre_b = vec(-0.5, 0.5) if has_z and norm == "layer" else None
    act = gate if gate in ("silu", "sigmoid") else "none"
    g = g64 = None
    if gate == "channel":
        g64 = vec(-1, 1)
        g = f32_dev(g64)
    elif gate != "none":
        g, g64 = rand((m, n), dtype, 4, -9, 9)
    if extra:
        x = strided(x, extra)
        r = strided(r, 2 * extra) if has_res else None
        g = strided(g, extra) if g is not None and g.dim() == 2 else g
    dev = lambda a: None if a is None else f32_dev(a)  # noqa: E731
    y = strided(sentinel((m, n), dtype), extra) if has_y else None
    z = strided(sentinel((m, n), dtype), extra) if has_z else None
    op = ops.block_norm(x, y, residual=r, post=dev(post), post_bias=dev(post_b), gate=g, gate_act=act, scale=scale, z=z,
                        pre=dev(pre), pre_bias=dev(pre_b), norm=norm)
    op.run()
    torch.cuda.synchronize()
    s32 = float(np.float32(scale))
    wy, wz, ey, ez = seq.block_norm(x64, r64, post, post_b, g64, act, s32, pre, pre_b, norm, float(np.float32(1e-5)),
                                    seq.HALF_STEP[dtype])
    if has_y:
        _inside(to_f64(y), wy, ey, "y")
    if has_z:
        _inside(to_f64(z), wz, ez, "z")
    elastic_bitwise(op, [t for t in (y, z) if t is not None], orc, bits)
    if extra:  # what lies between the rows is left alone
        for t in (y, z):
            if t is not None:
                assert torch.isnan(t.as_strided((m, extra), (n + extra, 1), n)).all()


def test_block_norm_of_large_and_zero_rows(ops, seq):
    x = torch.zeros((3, 4096), dtype=torch.float32, device="cuda")
    x[1] = 1e18
    x[2] = 3e-30
    w = torch.ones(4096, device="cuda")
    z = torch.empty_like(x)
    ops.block_norm(x, z=z, pre=w).run()
    torch.cuda.synchronize()
    z = to_f64(z)
    assert np.all(z[0] == 0) and np.allclose(z[1], 1.0, rtol=1e-5) and np.allclose(z[2], 3e-30 / np.sqrt(1e-5), rtol=1e-5)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n", [(6000, 768), (1100, 4096), (260, 16640), (5003, 1001)])
def test_block_norm_of_more_than_the_caches_hold(ops, orc, dtype, m, n):
    """Large ops move their rows past the caches: the bits of small ones over the same rows."""
    x, r, g = (rand((m, n), dtype, 30 + i)[0] for i in range(3))
    w = [f32_dev(np.random.default_rng(33 + i).uniform(-1, 1, n)) for i in range(2)]
    y, z = sentinel((m, n), dtype), sentinel((m, n), dtype)
    make = lambda a, b: ops.block_norm(x[a:b], y[a:b], residual=r[a:b], post=w[0], gate=g[a:b], gate_act="silu", z=z[a:b], pre=w[1])  # noqa: E731
    op = make(0, m)
    assert 5 * m * n * x.element_size() > 32e6
    ref = elastic_bitwise(op, [y, z], orc, bits, plans=(1, 3), blocks=(64, 256))
    y.fill_(-77.0)
    z.fill_(-77.0)
    for a in range(0, m, 251):
        make(a, min(m, a + 251)).run()
    torch.cuda.synchronize()
    assert [bits(y), bits(z)] == ref


# ---------------------------------------------------------------------- rotary
ROTARY_CASES = [
    # new, ctx, heads, kv_heads, d, rot, page, token_major, interleaved, scale
    ([1], [129], 12, 12, 64, 64, 16, False, False, 1.0),
    ([1, 1, 1], [1, 70000, 1000000], 8, 2, 128, 128, 64, True, False, 1.25),
    ([5, 0, 17, 1], [5, 40, 33, 16], 6, 3, 128, 64, 16, True, True, 1.0),
    ([3, 2], [9, 2], 4, 1, 80, 80, 7, False, False, 1.0),
    ([3, 2], [9, 2], 4, 1, 80, 40, 7, False, True, 1.0),     # the turned part is no whole vectors
    ([4], [6], 2, 1, 30, 6, 4, True, False, 1.0),            # odd sizes throughout
    ([4], [6], 2, 1, 7, 4, 3, False, True, 0.5),             # an odd head
    ([6], [6], 3, 2, 256, 256, 5, False, True, 1.0),
    ([2], [4], 2, 2, 16, 0, 2, False, False, 1.0),           # nothing is turned
    ([1] * 70, list(range(1, 71)), 4, 2, 64, 64, 16, False, False, 1.0),   # more sequences than lanes
    ([700], [900], 8, 1, 64, 32, 32, False, False, 1.0),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("case", ROTARY_CASES)
def test_rotary_and_append(ops, seq, orc, dtype, case):
    new, ctx, heads, kv, d, rot, page, token_major, inter, scale = case
    # pages of the older tokens are not needed: only those of new tokens are there
    b = Batch(new, [min(c, 2048) for c in ctx], page, kv, d, dtype, 11, token_major)
    if max(ctx) > 2048:
        b.table = np.full((len(ctx), -(-max(ctx) // page)), -1, dtype=np.int32)
        for s, c in enumerate(ctx):
            b.table[s, (c - 1) // page] = s
        b.kv_len = np.array(ctx, dtype=np.int32)
    b.k.fill_(-77.0)
    b.v.fill_(-77.0)
    x, x64 = rand((b.tokens, (heads + 2 * kv) * d), dtype, 12, -2, 2)
    freq = ops.rotary_freqs(rot, 10000.0, 4.0, 64) if rot else torch.empty(0, dtype=torch.float64)
    y = sentinel((b.tokens, heads * d), dtype)
    q_start, kv_len, table = b.arrays()
    op = ops.rotary(x, y, freq.cuda(), q_start, kv_len, heads=heads, head_dim=d, kv_heads=kv, k_cache=b.k, v_cache=b.v,
                    page_table=table, interleaved=inter, scale=scale)
    op.run()
    torch.cuda.synchronize()
    q, kv_at = seq.rotary(x64, freq.numpy(), b.q_start, b.kv_len, heads, kv, d, b.table, page, b.pages, inter, scale)
    h = seq.HALF_STEP[dtype]
    gy, gk, gv = to_f64(y), to_f64(b.k), to_f64(b.v)
    written = np.zeros((b.pages, page), dtype=bool)
    for r in range(b.tokens):
        if r in q:
            _inside(gy[r], q[r][0], q[r][1] * (1 + h) + h * np.abs(q[r][0]) + 2.0 ** -25, r)
        else:
            assert np.all(gy[r] == -77.0), r
    for (p, s), (kk, ke, vv) in kv_at.items():
        written[p, s] = True
        _inside(gk[p, :, s], kk, ke * (1 + h) + h * np.abs(kk) + 2.0 ** -25, ("key", p, s))
        assert np.array_equal(gv[p, :, s], vv)
    for g in (gk, gv):
        assert np.all(g.transpose(0, 2, 1, 3)[~written] == -77.0)
    assert len(kv_at) == sum(new)
    elastic_bitwise(op, [y, b.k, b.v], orc, bits)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("inter,d", [(False, 128), (True, 128), (False, 90)])
def test_rotary_of_more_than_the_caches_hold(ops, orc, dtype, inter, d):
    """Large ops move their rows past the caches: the bits of small ones over the same tokens."""
    heads, kv, new = 24, 4, [2000, 1, 999]
    b = Batch(new, [2500, 1, 1000], 16, kv, d, dtype, 25, behind=0)
    x, _ = rand((b.tokens, (heads + 2 * kv) * d), dtype, 26)
    y = sentinel((b.tokens, heads * d), dtype)
    q_start, kv_len, table = b.arrays()
    freq = ops.rotary_freqs(d // 2 * 2).cuda()
    op = ops.rotary(x, y, freq, q_start, kv_len, heads=heads, head_dim=d, kv_heads=kv, k_cache=b.k, v_cache=b.v, page_table=table,
                    interleaved=inter)
    assert 2 * x.numel() * x.element_size() > 32e6
    ref = elastic_bitwise(op, [y, b.k, b.v], orc, bits, plans=(1, 3), blocks=(64, 256))
    for t in (y, b.k, b.v):
        t.fill_(-77.0)
    at = 0
    for s, n in enumerate(new):                # pieces of a sequence's tokens, each at the end of its cache
        for i in range(0, n, 500):
            m = min(500, n - i)
            part = torch.tensor([0, m], dtype=torch.int32, device="cuda")
            length = torch.tensor([b.ctx[s] - n + i + m], dtype=torch.int32, device="cuda")
            ops.rotary(x[at:at + m], y[at:at + m], freq, part, length, heads=heads, head_dim=d, kv_heads=kv, k_cache=b.k,
                       v_cache=b.v, page_table=table[s:s + 1], interleaved=inter).run()
            at += m
    torch.cuda.synchronize()
    assert [bits(t) for t in (y, b.k, b.v)] == ref


@pytest.mark.parametrize("dtype", DTYPES)
def test_rotary_without_cache_and_into_columns_of_one_buffer(ops, seq, dtype):
    buf = torch.full((9, 5 * 64), -77.0, dtype={"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype], device="cuda")
    x, x64 = rand((9, 2 * 64), dtype, 5)
    buf[:, :128] = x
    freq = ops.rotary_freqs(64)
    q_start, kv_len = torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda"), torch.tensor([4, 2], dtype=torch.int32, device="cuda")
    ops.rotary(buf[:, :128], buf[:, 192:], freq.cuda(), q_start, kv_len, heads=2, head_dim=64).run()
    torch.cuda.synchronize()
    got = to_f64(buf)
    q, _ = seq.rotary(x64, freq.numpy(), q_start.cpu().numpy(), kv_len.cpu().numpy(), 2, 0, 64)  # positions -2 .. among them
    h = seq.HALF_STEP[dtype]
    for r in range(8):
        _inside(got[r, 192:], q[r][0], q[r][1] * (1 + h) + h * np.abs(q[r][0]) + 2.0 ** -25, r)
    assert np.array_equal(got[:, :128], x64) and np.all(got[:, 128:192] == -77.0) and np.all(got[8, 192:] == -77.0)


def test_tokens_without_a_place_are_not_stored(ops):
    """Negative positions, absent pages and positions behind the page table: queries are turned, nothing is stored."""
    b = Batch([4, 3, 2], [2, 40, 16], 8, 1, 64, "f16", 21, absent=[(1, 4, -1), (2, 1, 999)], beyond=0)
    b.k.fill_(-77.0)
    b.v.fill_(-77.0)
    x, _ = rand((b.tokens, 3 * 64), "f16", 22)
    y = sentinel((b.tokens, 64), "f16")
    q_start, kv_len, table = b.arrays()
    ops.rotary(x, y, ops.rotary_freqs(64).cuda(), q_start, kv_len, heads=1, head_dim=64, kv_heads=1, k_cache=b.k, v_cache=b.v,
               page_table=table).run()
    torch.cuda.synchronize()
    stored = (to_f64(b.v)[:, 0, :, 0] != -77.0).sum()
    assert stored == 2                      # the two of sequence 0 at positions 0 and 1
    assert np.all(to_f64(y)[:9] != -77.0) and np.all(to_f64(y)[9:] == -77.0)


# ------------------------------------------------------------------- attention
ATTEND_CASES = [
    # new, ctx, heads, kv_heads, d, page, token_major, window, causal
    ([1], [1], 1, 1, 64, 16, False, 0, True),
    ([1], [129], 12, 12, 64, 16, False, 0, True),
    ([1, 1, 0, 1], [7, 300, 40, 1025], 8, 2, 128, 16, True, 0, True),
    ([1] * 70, [1 + 13 * i % 97 for i in range(70)], 4, 1, 64, 16, False, 0, True),
    ([1] * 3, [5000, 1, 129], 16, 1, 128, 64, False, 0, True),
    ([1, 1], [900, 333], 5, 1, 80, 24, True, 100, True),
    ([2, 3, 1], [50, 200, 64], 8, 2, 128, 3, False, 0, True),      # several rows of a head group, a page ends anywhere
    ([4, 2], [130, 31], 2, 2, 8, 1, False, 5, True),               # pages of one token, the smallest head
    ([3], [3], 3, 1, 256, 16, False, 0, True),
    ([1, 1], [700, 20], 2, 1, 136, 32, True, 0, True),
    ([3, 2], [40, 7], 4, 2, 64, 16, False, 0, False),              # every key for every token
    ([17], [17], 1, 1, 64, 16, False, 0, True),
    ([40, 1, 0, 65], [40, 90, 12, 300], 4, 2, 128, 16, False, 0, True),
    ([128], [128], 2, 2, 64, 64, True, 0, True),
    ([129, 200], [129, 1000], 6, 2, 96, 24, True, 0, True),
    ([300], [1300], 1, 1, 128, 32, False, 0, True),                # divided keys
    ([150, 33], [500, 33], 5, 1, 40, 16, False, 70, True),         # window, an odd group
    ([64, 30], [64, 200], 2, 1, 256, 16, False, 0, True),
    ([50], [170], 4, 4, 200, 16, True, 0, False),
    ([90, 40], [90, 300], 8, 8, 72, 100, False, 33, False),
]


def _attend(ops, b, dtype, heads, d, window, causal, max_q, extra=0, seed=31):
    x, x64 = rand((b.tokens, heads * d), dtype, seed, -2, 2)
    y = sentinel((b.tokens, heads * d), dtype)
    if extra:
        x, y = strided(x, extra), strided(y, extra)
    q_start, kv_len, table = b.arrays()
    op = ops.attention(x, b.k, b.v, y, q_start, kv_len, table, heads=heads, window=window, causal=causal, max_q=max_q)
    return op, x64, y


def _p_step(seq, dtype, rows):
    """Probabilities are rounded once in the kernel for many rows, and to a sum of two numbers in the other."""
    h = seq.HALF_STEP[dtype]
    return 2 * h * h if rows else 2 * h


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("case", ATTEND_CASES)
def test_attention(ops, seq, orc, dtype, case):
    new, ctx, heads, kv, d, page, token_major, window, causal = case
    b = Batch(new, ctx, page, kv, d, dtype, 30, token_major).hide_unused()
    few = max(new) * (heads // kv) <= 16
    # whether a caller knows its longest sequence must not matter for what comes out
    for max_q in (max(new), None):
        op, x64, y = _attend(ops, b, dtype, heads, d, window, causal, max_q, extra=8)
        op.run()
        torch.cuda.synchronize()
        want = seq.attention(x64, b.k64, b.v64, b.q_start, b.kv_len, b.table, heads, None, causal, window, None,
                             seq.HALF_STEP[dtype], _p_step(seq, dtype, few and max_q is not None))
        got = to_f64(y)
        for r in range(b.tokens):
            if r in want:
                _inside(got[r], want[r][0], want[r][1], (max_q, r))
            else:
                assert np.all(got[r] == -77.0), r
        elastic_bitwise(op, [y], orc, bits, plans=(1, 3, 8) if max_q else (2,))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,ctx", [([1, 1], [9000, 20000]), ([5], [12000])])
def test_attention_over_long_caches(ops, seq, orc, dtype, new, ctx):
    """Many tiles share each output."""
    b = Batch(new, ctx, 64, 2, 128, dtype, 40).hide_unused()
    op, x64, y = _attend(ops, b, dtype, 8, 128, 0, True, max(new))
    assert op.info.ksplit > 1
    op.run()
    torch.cuda.synchronize()
    want = seq.attention(x64, b.k64, b.v64, b.q_start, b.kv_len, b.table, 8, half_step=seq.HALF_STEP[dtype],
                         p_step=_p_step(seq, dtype, max(new) * 4 <= 16))
    got = to_f64(y)
    for r, (w, e) in want.items():
        _inside(got[r], w, e, r)
    elastic_bitwise(op, [y], orc, bits)


DIVISIONS = [
    # new, ctx, heads, kv_heads, d, page, token_major, window, max_q: how the work is divided among tiles
    ([20] * 70, [20 + 37 * i % 900 for i in range(70)], 8, 8, 64, 16, False, 0, None),     # more row tiles than run at once
    ([130] * 9 + [1], [130 + 50 * i for i in range(9)] + [30000], 64, 32, 64, 32, False, 0, None),  # one very long sequence beside them
    ([1, 300, 1, 77, 1, 1], [3000, 700, 50, 4000, 1, 2047], 10, 5, 128, 24, True, 1500, None),  # single tokens beside chunks
    ([513], [9000], 4, 1, 128, 16, False, 0, None),                                        # one chunk, one cache head
    ([40, 3], [40, 60000], 2, 1, 64, 64, False, 0, None),                                  # as many parts as can be joined
    ([2100], [2100], 32, 32, 64, 64, False, 0, None),                                      # a tile for each
    ([1] * 200, [1 + 11 * i % 700 for i in range(200)], 8, 4, 64, 16, False, 0, 1),        # single tokens of many sequences
    ([1, 1, 1], [40000, 3, 129], 2, 1, 128, 64, False, 0, 1),                              # joined in two stages
    ([1, 300, 1, 77, 1, 1], [3000, 700, 50, 4000, 1, 2047], 10, 5, 80, 24, True, 1500, None),  # heads of whole 32s but the last
    ([513], [9000], 4, 1, 96, 18, False, 0, None),                                         # pages that no load divides
    # several sequences to a lane that looks for a tile's work
    ([i % 50 for i in range(200)], [i % 50 + 3 * i % 90 for i in range(200)], 16, 4, 64, 16, False, 0, None),
    ([0] * 90 + [30, 1] + [0] * 60 + [7] * 3, [5] * 90 + [2500, 40] + [0] * 60 + [700, 7, 1300], 8, 2, 64, 16, False, 0, None),
    ([i % 2 for i in range(330)], [i % 2 + 5 * i % 700 for i in range(330)], 8, 2, 64, 16, True, 0, 1),
    ([0] * 100 + [2, 1] + [1, 0] * 40, [0] * 100 + [9000, 300] + [130, 9] * 40, 2, 1, 128, 32, False, 0, 2),
]


@pytest.mark.parametrize("case", DIVISIONS)
def test_attention_however_the_work_is_divided(ops, seq, orc, case):
    new, ctx, heads, kv, d, page, token_major, window, max_q = case
    b = Batch(new, ctx, page, kv, d, "f16", 35, token_major).hide_unused()
    op, x64, y = _attend(ops, b, "f16", heads, d, window, True, max_q)
    ref = elastic_bitwise(op, [y], orc, bits, plans=(1, 5))
    for _ in range(2):                         # counters are back at zero
        y.fill_(-77.0)
        op.run()
        torch.cuda.synchronize()
        assert [bits(y)] == ref
    step = max(1, sum(new) // 60)              # rows compared: every step-th
    want = seq.attention(x64, b.k64, b.v64, b.q_start, b.kv_len, b.table, heads, window=window, half_step=seq.HALF_STEP["f16"],
                         p_step=_p_step(seq, "f16", max_q == 1), stride=step)
    got = to_f64(y)
    for r, (w, e) in want.items():
        _inside(got[r], w, e, r)
    assert np.all(got[sum(new):] == -77.0) and np.all(got[:sum(new)] != -77.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,heads", [([4, 2], 4), ([200, 2], 4)])
def test_rows_without_keys_give_zeros(ops, seq, dtype, new, heads):
    """More new tokens than keys, absent pages, an empty cache: rows that see nothing are zero, the others right."""
    b = Batch(new, [150 if new[0] > 16 else 3, 0], 16, 2, 64, dtype, 50, absent=[(0, 0, -1)]).hide_unused()
    op, x64, y = _attend(ops, b, dtype, heads, 64, 0, True, None if new[0] > 16 else 8)
    op.run()
    torch.cuda.synchronize()
    want = seq.attention(x64, b.k64, b.v64, b.q_start, b.kv_len, b.table, heads, half_step=seq.HALF_STEP[dtype],
                         p_step=_p_step(seq, dtype, False))
    got = to_f64(y)
    zero = [r for r in want if not want[r][0].any()]
    assert len(zero) >= 3
    for r, (w, e) in want.items():
        _inside(got[r], w, e, r)
        assert r not in zero or not got[r].any()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("window", [0, 6])
@pytest.mark.parametrize("n,ctx,heads", [(4, 20, 4), (4, 300, 4), (70, 70, 2), (140, 400, 1)])
def test_what_a_row_does_not_see_never_reaches_it(ops, seq, dtype, n, ctx, heads, window):
    """Infinities and NaN in the keys and values of tokens that some rows see and others do not."""
    b = Batch([n], [ctx], 16, 1, 64, dtype, 60, behind=0)
    last, first = ctx - 1, ctx - n
    bad = {last: float("nan"), last - 2: float("inf"), first + 1: float("-inf")}
    for j, value in bad.items():
        p, s = int(b.table[0, j // 16]), j % 16
        b.v[p, 0, s, 3] = value
        b.v[p, 0, s, 40] = value
        b.v64[p, 0, s, 3] = b.v64[p, 0, s, 40] = value
    p, s = int(b.table[0, last // 16]), last % 16
    b.k[p, 0, s] = float("nan")
    b.k64[p, 0, s] = np.nan
    op, x64, y = _attend(ops, b, dtype, heads, 64, window, True, n)
    op.run()
    torch.cuda.synchronize()
    got = to_f64(y)
    with np.errstate(invalid="ignore"):
        want = seq.attention(x64, b.k64, b.v64, b.q_start, b.kv_len, b.table, heads, window=window,
                             half_step=seq.HALF_STEP[dtype], p_step=_p_step(seq, dtype, False))
    for r, (w, e) in want.items():
        pos = first + r
        seen = [v for j, v in bad.items() if j <= pos and (not window or j > pos - window)]
        rows, gr = w.reshape(heads, 64), got[r].reshape(heads, 64)
        if pos == last:                      # its own key is NaN
            assert np.all(np.isnan(gr)), r
            continue
        for dd in range(64):
            if dd in (3, 40) and seen:
                assert np.array_equal(np.isnan(gr[:, dd]), np.isnan(rows[:, dd])), (r, dd)
                assert np.array_equal(np.sign(gr[:, dd][~np.isnan(gr[:, dd])]), np.sign(rows[:, dd][~np.isnan(rows[:, dd])]))
                assert not np.any(np.isfinite(gr[:, dd]))
            else:
                _inside(gr[:, dd], rows[:, dd], e.reshape(heads, 64)[:, dd], (r, dd))


def test_max_q_leaves_later_rows_alone(ops):
    b = Batch([6, 1], [40, 9], 16, 1, 64, "f16", 70)
    _, _, whole = _attend(ops, b, "f16", 2, 64, 0, True, 6)
    op, _, whole = _attend(ops, b, "f16", 2, 64, 0, True, 6)
    op.run()
    op2, _, part = _attend(ops, b, "f16", 2, 64, 0, True, 4)
    op2.run()
    torch.cuda.synchronize()
    assert bits(whole[:4]) == bits(part[:4]) and bits(whole[6:7]) == bits(part[6:7])
    assert (part[4:6] == -77.0).all() and (part[7:] == -77.0).all()


def test_attention_over_the_encoders_projection(ops, seq):
    """Keys and values as they lie in the encoder's qkv rows, one page per sequence: its three operators' result."""
    B, S, H, D = 2, 70, 12, 64
    qkv, q64 = rand((B * S, 3 * H * D), "bf16", 80, -1, 1)
    cut = lambda i: qkv.view(B, S, 3, H, D)[:, :, i].permute(0, 2, 1, 3)  # noqa: E731
    y = sentinel((B * S, H * D), "bf16")
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    op = ops.attention(qkv[:, :H * D], cut(1), cut(2), y, ints([0, S, 2 * S]), ints([S, S]), ints([[0], [1]]), heads=H, causal=False)
    op.run()
    torch.cuda.synchronize()
    kv = q64.reshape(B, S, 3, H, D).transpose(2, 0, 3, 1, 4)
    want = seq.attention(q64[:, :H * D], np.ascontiguousarray(kv[1]), np.ascontiguousarray(kv[2]), [0, S, 2 * S], [S, S],
                         np.array([[0], [1]]), H, causal=False, half_step=seq.HALF_STEP["bf16"], p_step=_p_step(seq, "bf16", False))
    for r, (w, e) in want.items():
        _inside(to_f64(y)[r], w, e, r)


# ------------------------------------------------------- lengths of a later call
def _replayed(op, y, arrays, batches, eager):
    """A captured pass, replayed with each batch's arrays, gives the eager pass's bits, with other work between."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        op.run()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        op.run()
    for _ in range(2):
        for i, vals in enumerate(batches):
            for t, v in zip(arrays, vals):
                t.copy_(v)
            y.fill_(-77.0)
            junk = torch.randn(1 << 18, device="cuda")
            float((junk * 2).sum())
            g.replay()
            torch.cuda.synchronize()
            assert bits(y) == eager[i], i


@pytest.mark.parametrize("max_q", [2, None])
def test_graph_replays_with_other_lengths(ops, max_q):
    """One operator serves batches of any lengths within its capacities; none of them finds counters of another."""
    sets = [([1, 1, 1], [2000, 3, 900]), ([2, 0, 1], [2, 60, 2047]), ([0, 0, 0], [5, 5, 5]), ([1, 2, 1], [64, 64, 1])]
    b = Batch([1, 1, 1], [2048, 2048, 2048], 16, 2, 128, "bf16", 90)
    x, _ = rand((5, 8 * 128), "bf16", 91)
    y = sentinel((5, 8 * 128), "bf16")
    q_start, kv_len, table = b.arrays()
    op = ops.attention(x, b.k, b.v, y, q_start, kv_len, table, heads=8, max_q=max_q)
    assert op.info.ksplit > 1
    batches = [(torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32), torch.tensor(c, dtype=torch.int32)) for n, c in sets]
    eager = []
    for vals in batches:
        q_start.copy_(vals[0])
        kv_len.copy_(vals[1])
        y.fill_(-77.0)
        op.run()
        torch.cuda.synchronize()
        eager.append(bits(y))
    assert len(set(eager)) == len(sets)
    _replayed(op, y, (q_start, kv_len), batches, eager)


def test_wild_arrays_stay_inside(ops):
    """Starts, lengths and pages of any value are clamped or absent: what comes out is finite or left alone."""
    b = Batch([1, 1, 1, 1], [64, 64, 64, 64], 16, 1, 64, "f16", 95)
    big, low = 2 ** 31 - 1, -2 ** 31
    for max_q in (1, None):
        for starts, lens, pages in [([0, 1, 2, 3, 4], [big, low, -1, 70], None), ([big, low, 3, 1, big], [64] * 4, None),
                                    ([-5, 2, 1, 9, 2], [10] * 4, None), ([0, 1, 2, 3, 4], [64] * 4, [big, low, -1, 10 ** 6])]:
            x, _ = rand((6, 2 * 64), "f16", 96)
            y = sentinel((6, 2 * 64), "f16")
            q_start, kv_len, table = b.arrays()
            q_start.copy_(torch.tensor(starts, dtype=torch.int32))
            kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
            if pages:
                table[:, 0] = torch.tensor(pages, dtype=torch.int32)
            xr, _ = rand((6, 4 * 64), "f16", 97)
            yr = sentinel((6, 2 * 64), "f16")
            kc, vc = b.k.clone(), b.v.clone()
            ops.rotary(xr, yr, ops.rotary_freqs(64).cuda(), q_start, kv_len, heads=2, head_dim=64, kv_heads=1, k_cache=kc,
                       v_cache=vc, page_table=table).run()
            ops.attention(x, b.k, b.v, y, q_start, kv_len, table, heads=2, max_q=max_q).run()
            torch.cuda.synchronize()
            assert torch.isfinite(y).all() and torch.isfinite(yr).all() and torch.isfinite(kc).all()


def test_noalloc_attention_matches(ops):
    from paper_2307_04339_amd import _lib as L
    for max_q, new, ctx in [(1, [1, 1], [5000, 700]), (None, [40, 3], [2500, 900])]:
        b = Batch(new, ctx, 32, 2, 64, "f16", 98)
        op, _, y = _attend(ops, b, "f16", 8, 64, 0, True, max_q)
        op.run()
        torch.cuda.synchronize()
        ref = bits(y)
        h = ctypes.c_void_p()
        assert L.load().miriam_seq_op_create_noalloc(ctypes.byref(op.desc), ctypes.byref(h)) == 0
        y.fill_(-77.0)
        assert L.load().miriam_op_run(h, ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        torch.cuda.synchronize()
        info = L.OpInfo()
        L.load().miriam_op_query(h, ctypes.byref(info))
        assert info.ksplit > 1 and bits(y) == ref
        assert L.load().miriam_op_destroy(h) == 0


def test_another_stream(ops):
    b = Batch([1, 1], [900, 77], 16, 2, 128, "bf16", 99)
    op, _, y = _attend(ops, b, "bf16", 8, 128, 0, True, 1)
    op.run()
    torch.cuda.synchronize()
    ref = bits(y)
    y.fill_(-77.0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    op.run(s)
    s.synchronize()
    assert bits(y) == ref


def test_one_graph_over_every_division(ops):
    """A chunk in pieces, runs of a list, a tile per row tile, single tokens: one captured op, batch after batch."""
    heads, d, seqs, ctx = 32, 64, 70, 20000
    x, _ = rand((2200, heads * d), "bf16", 200, -2, 2)
    pages = 700
    k, v = (rand((pages, heads, 32, d), "bf16", 201 + i)[0] for i in range(2))
    table = torch.from_numpy(np.random.default_rng(203).integers(0, pages, (seqs, ctx // 32)).astype(np.int32)).cuda()
    y = sentinel((2200, heads * d), "bf16")
    zero = [0] * seqs
    sets = [([1000] + zero[1:], [6000] + zero[1:]), ([1] * 60 + [300, 300] + zero[62:], [40] * 61 + [ctx] + zero[62:]),
            ([30] * 70, [40 + i for i in range(70)]), ([1] * 70, [1 + i for i in range(70)]), (zero, [7] * 70)]
    batches = [(torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32), torch.tensor(c, dtype=torch.int32)) for n, c in sets]
    q_start, kv_len = (t.cuda() for t in batches[0])
    op = ops.attention(x, k, v, y, q_start, kv_len, table, heads=heads)
    assert op.info.ksplit > 1
    eager = []
    for vals in batches:
        q_start.copy_(vals[0])
        kv_len.copy_(vals[1])
        y.fill_(-77.0)
        ops.attention(x, k, v, y, q_start, kv_len, table, heads=heads).run()   # (its workspace is its own)
        torch.cuda.synchronize()
        eager.append(bits(y))
    assert len(set(eager)) == len(sets)
    _replayed(op, y, (q_start, kv_len), batches, eager)


@pytest.mark.parametrize("max_q", [1, None])
def test_two_operators_at_once(ops, max_q):
    """Operators of their own workspaces on two streams, over the same caches."""
    new, ctx = ([1] * 6, [9000, 40, 5000, 7000, 1, 333]) if max_q else ([200, 1, 70], [8000, 3000, 70])
    b = Batch(new, ctx, 32, 2, 128, "f16", 210)
    made = [_attend(ops, b, "f16", 8, 128, 0, True, max_q, seed=211 + i) for i in range(2)]
    ref = []
    for op, _, y in made:
        op.run()
        torch.cuda.synchronize()
        ref.append(bits(y))
        y.fill_(-77.0)
    assert ref[0] != ref[1] and made[0][0].info.ksplit > 1
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for (op, _, _), s in zip(made, streams):
            op.run(s)
    torch.cuda.synchronize()
    assert [bits(y) for _, _, y in made] == ref


# -------------------------------------------------- the operators one after another
class Layer:
    """A decoder layer's step over a paged cache: norms, projections, rotary and append, attention, gated block."""

    def __init__(self, ops, b, dtype, heads, kv, d, seed):
        hid, T = heads * d, b.tokens
        self.b, self.heads, self.kv, self.d, self.dtype = b, heads, kv, d, dtype
        r = lambda shape, i, s: rand(shape, dtype, seed + i, -s, s)  # noqa: E731
        self.x, self.x64 = r((T, hid), 0, 1.0)
        self.wqkv, self.wqkv64 = r(((heads + 2 * kv) * d, hid), 1, hid ** -0.5)
        self.wo, self.wo64 = r((hid, hid), 2, hid ** -0.5)
        rng = np.random.default_rng(seed)
        self.n1, self.post, self.n2 = (rng.uniform(0.5, 1.5, hid).astype(np.float32).astype(np.float64) for _ in range(3))
        self.freq = ops.rotary_freqs(d)
        buf = lambda n: sentinel((T, n), dtype)  # noqa: E731
        self.h1, self.qkv, self.q, self.ctx, self.o, self.y, self.z = buf(hid), buf((heads + 2 * kv) * d), buf(hid), buf(hid), buf(hid), buf(hid), buf(hid)
        self.q_start, self.kv_len, self.table = b.arrays()
        self.ops = [
            ops.block_norm(self.x, z=self.h1, pre=f32_dev(self.n1)),
            ops.gemm(self.h1, self.wqkv, self.qkv),
            ops.rotary(self.qkv, self.q, self.freq.cuda(), self.q_start, self.kv_len, heads=heads, head_dim=d, kv_heads=kv,
                       k_cache=b.k, v_cache=b.v, page_table=self.table),
            ops.attention(self.q, b.k, b.v, self.ctx, self.q_start, self.kv_len, self.table, heads=heads, max_q=max(b.new)),
            ops.gemm(self.ctx, self.wo, self.o),
            ops.block_norm(self.o, self.y, residual=self.x, post=f32_dev(self.post), scale=0.5, z=self.z, pre=f32_dev(self.n2)),
        ]
        self.outs = [self.h1, self.qkv, self.q, self.ctx, self.o, self.y, self.z]

    def run(self):
        for op in self.ops:
            op.run()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("new,ctx", [([1, 1, 1], [40, 300, 7]), ([33, 1, 90], [33, 200, 120])])
def test_a_decoder_layers_step(ops, seq, dtype, new, ctx):
    heads, kv, d = 8, 2, 64
    b = Batch(new, ctx, 16, kv, d, dtype, 110, behind=0)
    l = Layer(ops, b, dtype, heads, kv, d, 111)
    l.run()
    torch.cuda.synchronize()
    # each operator against float64 on the inputs that it had: the caches hold the new keys and values now
    h = seq.HALF_STEP[dtype]
    got = {n: to_f64(getattr(l, n)) for n in ("h1", "qkv", "q", "ctx", "o", "y", "z")}
    _, w, _, e = seq.block_norm(l.x64, pre=l.n1, half_step=h)
    _inside(got["h1"], w, e, "first norm")
    q, kv_at = seq.rotary(got["qkv"], l.freq.numpy(), b.q_start, b.kv_len, heads, kv, d, b.table, 16, b.pages)
    k64, v64 = to_f64(b.k), to_f64(b.v)
    for r in q:
        _inside(got["q"][r], q[r][0], q[r][1] * (1 + h) + h * np.abs(q[r][0]) + 2.0 ** -25, r)
    for (p, s), (kk, ke, vv) in kv_at.items():
        _inside(k64[p, :, s], kk, ke * (1 + h) + h * np.abs(kk) + 2.0 ** -25, (p, s))
        assert np.array_equal(v64[p, :, s], vv)
    at = seq.attention(got["q"], k64, v64, b.q_start, b.kv_len, b.table, heads, half_step=h, p_step=_p_step(seq, dtype, False))
    for r, (w, e) in at.items():
        _inside(got["ctx"][r], w, e, r)
    wy, wz, ey, ez = seq.block_norm(got["o"], l.x64, l.post, scale=0.5, pre=l.n2, half_step=h)
    _inside(got["y"], wy, ey, "y")
    _inside(got["z"], wz, ez, "z")


@pytest.mark.parametrize("policy,graphs", [("elastic", 1), ("elastic", 0), ("multistream", 1)])
def test_decoder_steps_as_tasks_of_the_coordinator(ops, policy, graphs):
    """A batch of single tokens as critical requests beside chunks of prompts as best-effort ones, cut into shards:
    every output is bitwise the eager pass's, with other lengths after a while."""
    from paper_2307_04339_amd.runtime import Coordinator
    crit = Layer(ops, Batch([1] * 4, [400, 30, 1200, 1], 16, 2, 64, "f16", 120, behind=0), "f16", 8, 2, 64, 121)
    best = Layer(ops, Batch([200, 70], [900, 70], 16, 2, 128, "bf16", 130, behind=0), "bf16", 8, 2, 128, 131)
    lens = [[400, 30, 1200, 1], [401, 31, 1201, 2], [9, 1000, 64, 129]]

    def eager():
        for l in (crit, best):
            l.run()
        torch.cuda.synchronize()
        return [bits(t) for l in (crit, best) for t in l.outs]

    with Coordinator(policy=policy, graphs=graphs, profile_reps=1, n_be_streams=1, inflight_depth=2, quantum_us=20.0) as co:
        tc, tb = co.task(crit.ops), co.task(best.ops)
        for n in lens:
            n = [min(v, int(crit.b.table.shape[1]) * 16) for v in n]
            crit.kv_len.copy_(torch.tensor(n, dtype=torch.int32))
            ref = eager()
            for l in (crit, best):
                for t in l.outs:
                    t.fill_(-77.0)
            torch.cuda.synchronize()
            tickets = {co.submit(tb, False), co.submit(tc, True)}
            co.drain(60000)
            recs = {r.ticket: r for r in co.poll()}
            assert set(recs) == tickets and all(r.status == 0 for r in recs.values())
            torch.cuda.synchronize()
            assert [bits(t) for l in (crit, best) for t in l.outs] == ref
