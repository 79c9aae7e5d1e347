"""Caches and rows whose offsets pass 32 bits: pages at the end of caches of more than 2^31 values, rows that lie 2^28
values apart."""
import numpy as np
import pytest
import torch

from gpu_util import TORCH, gpu_available, rand, to_f64

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]

PAGE, KV, D = 16, 2, 64
PAGES = (1 << 31) // (PAGE * KV * D) + 40


@pytest.fixture(scope="module")
def ops():
    from paper_2307_04339_amd import ops as o
    return o


@pytest.fixture(scope="module")
def seq():
    from oracle import sequences
    return sequences


@pytest.fixture(scope="module")
def far():
    """Two caches of 4.3 GB, not initialised; the pages in use are the last ones and the first ones."""
    made = [torch.empty((PAGES, KV, PAGE, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    yield made
    made.clear()
    torch.cuda.empty_cache()


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("new,max_q,rows_apart", [([1, 1], 1, 0), ([3, 2], None, 0), ([60, 9], None, 0), ([3, 2], 4, 1 << 28), ([20, 9], None, 1 << 26)])
def test_append_and_attention_far_behind(ops, seq, far, new, max_q, rows_apart):
    heads, ctx = 4, [70, 120]
    kc, vc = far
    table = np.array([[PAGES - 1 - i for i in range(8)], [PAGES - 20 - i if i % 2 else i for i in range(8)]], dtype=np.int32)
    used = np.unique(table)
    at = {int(p): i for i, p in enumerate(used)}
    small = np.vectorize(at.get)(table).astype(np.int32)         # the same pages in a cache of their own
    index = torch.from_numpy(used).cuda().long()
    (k, _), (v, _) = (rand((len(used), KV, PAGE, D), "bf16", 600 + i, -1.5, 1.5) for i in range(2))
    kc[index], vc[index] = k, v
    starts = np.concatenate([[0], np.cumsum(new)])
    m, width = sum(new), (heads + 2 * KV) * D
    x, x64 = rand((m, width), "bf16", 602, -2, 2)
    buf = None
    if rows_apart:
        buf = torch.empty((m - 1) * rows_apart + width, dtype=TORCH["bf16"], device="cuda")
        xr = buf.as_strided((m, width), (rows_apart, 1))
        xr.copy_(x)
        x = xr
    q, y = (torch.full((m, heads * D), -77.0, dtype=TORCH["bf16"], device="cuda") for _ in range(2))
    args = (_ints(starts), _ints(ctx))
    freq = ops.rotary_freqs(D)
    ops.rotary(x, q, freq.cuda(), *args, heads=heads, head_dim=D, kv_heads=KV, k_cache=kc, v_cache=vc, page_table=_ints(table)).run()
    torch.cuda.synchronize()
    h = seq.HALF_STEP["bf16"]
    wq, wkv = seq.rotary(x64, freq.numpy(), starts, ctx, heads, KV, D, small, PAGE, len(used))
    k64, v64, got = to_f64(kc[index]), to_f64(vc[index]), to_f64(q)
    assert len(wq) == m and len(wkv) == m
    for r, (w, e) in wq.items():
        assert np.all(np.abs(got[r] - w) <= e * (1 + h) + h * np.abs(w) + 2.0 ** -25), r
    for (p, s), (kk, ke, vv) in wkv.items():
        assert np.all(np.abs(k64[p, :, s] - kk) <= ke * (1 + h) + h * np.abs(kk) + 2.0 ** -25), (p, s)
        assert np.array_equal(v64[p, :, s], vv)
    ops.attention(q, kc, vc, y, *args, _ints(table), heads=heads, max_q=max_q).run()
    torch.cuda.synchronize()
    want = seq.attention(got, k64, v64, starts, ctx, small, heads, half_step=h, p_step=2 * h)
    out = to_f64(y)
    for r, (w, e) in want.items():
        assert np.all(np.abs(out[r] - w) <= e), r


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [64, 1000, 5000])
def test_norm_of_rows_far_apart(ops, seq, dtype, n):
    m, apart = 12, 1 << 28
    x, x64 = rand((m, n), dtype, 610, -2, 2)
    buf = torch.empty((m - 1) * apart + 2 * n + 8, dtype=TORCH[dtype], device="cuda")
    xr, zr = buf.as_strided((m, n), (apart, 1)), buf.as_strided((m, n), (apart, 1), n + 8)
    xr.copy_(x)
    zr.fill_(-77.0)
    w = np.random.default_rng(611).uniform(0.5, 1.5, n).astype(np.float32)
    ops.block_norm(xr, z=zr, pre=torch.from_numpy(w).cuda()).run()
    torch.cuda.synchronize()
    _, want, _, e = seq.block_norm(x64, pre=w.astype(np.float64), eps=float(np.float32(1e-5)), half_step=seq.HALF_STEP[dtype])
    assert np.all(np.abs(to_f64(zr) - want) <= e) and np.array_equal(to_f64(xr), x64)
