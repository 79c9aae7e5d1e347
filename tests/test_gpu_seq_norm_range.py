"""Block norms of rows whose squares, or their sums, lie beyond fp32, against float64."""
import numpy as np
import pytest
import torch

from gpu_util import bits, f32_dev, gpu_available, rand, to_f64
from seq_util import elastic_bitwise, sentinel

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]


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
    assert np.all(np.abs(got - want) <= bound), (what, float(np.max(np.abs(got - want) / bound)))


# A lane's values or a whole row's: every form of a row, whole vectors and ragged
SIZES = [(1e19, 4096), (1e18, 100000), (1e18, 16384), (3e37, 64), (3e37, 2050), (2e19, 1021), (1e25, 8192), (1e19, 20011), (3e37, 768)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("size,n", SIZES)
def test_block_norm_of_rows_beyond_the_range_of_squares(ops, seq, orc, dtype, norm, size, n):
    """Large rows among ordinary ones: of x alone, and of the sum with a large residual."""
    m = 6
    x, x64 = rand((m, n), dtype, 400, -1, 1)
    r, r64 = rand((m, n), dtype, 401, -1, 1)
    big = 2.0 ** np.floor(np.log2(size))                 # exact in either type
    for t, a, rows in ((x, x64, (1, 4)), (r, r64, (2, 4))):
        for i in rows:
            t[i] *= big
            a[i] *= big
    rng = np.random.default_rng(402)
    vec = lambda: rng.uniform(0.5, 1.5, n).astype(np.float32).astype(np.float64)  # noqa: E731
    post, pre = vec(), vec()
    b1, b2 = (vec(), vec()) if norm == "layer" else (None, None)
    dev = lambda a: None if a is None else f32_dev(a)  # noqa: E731
    h, eps = seq.HALF_STEP[dtype], float(np.float32(1e-5))
    for p in (post, None):
        y, z = sentinel((m, n), dtype), sentinel((m, n), dtype)
        pb = b1 if p is not None else None
        op = ops.block_norm(x, y, residual=r, post=dev(p), post_bias=dev(pb), z=z, pre=dev(pre), pre_bias=dev(b2), norm=norm)
        op.run()
        torch.cuda.synchronize()
        wy, wz, ey, ez = seq.block_norm(x64, r64, p, pb, scale=1.0, pre=pre, pre_bias=b2, norm=norm, eps=eps, half_step=h)
        _inside(to_f64(y), wy, ey, "y")
        _inside(to_f64(z), wz, ez, "z")
        elastic_bitwise(op, [y, z], orc, bits, plans=(1, 3))


@pytest.mark.parametrize("n", [1000, 5000, 20000])
def test_what_is_not_finite_stays_in_its_row(ops, n):
    x, _ = rand((4, n), "f32", 410)
    x[1, 3], x[2, n - 1] = float("inf"), float("nan")
    w = torch.ones(n, device="cuda")
    z, ref = torch.empty_like(x), torch.empty_like(x)
    ops.block_norm(x, z=z, pre=w).run()
    good = x.clone()
    good[1:3] = 1.0
    ops.block_norm(good, z=ref, pre=w).run()
    torch.cuda.synchronize()
    assert torch.equal(z[0], ref[0]) and torch.equal(z[3], ref[3])
    assert torch.isnan(z[1, 3]) and torch.isnan(z[2]).all()              # inf / inf
    assert (z[1].abs().nan_to_num(0.0) == 0).all()                       # and x / inf
