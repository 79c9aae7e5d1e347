"""fp16 results are rounded alike whatever the block: an affine sum and its rounding that the compiler makes one
instruction of, in some copies of a loop only, differ by a step in one of some 10^5 values, so millions are compared."""
import numpy as np
import pytest
import torch

from gpu_util import bits, empty, f32_dev, gpu_available, rand

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not gpu_available(), reason="needs an MI355X")]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,hw,c,k", [(16, 56, 64, 64), (24, 64, 16, 64)])
def test_resident_conv_with_affine_epilogue_in_every_block(dtype, n, hw, c, k):
    from paper_2307_04339_amd import _lib as L
    from paper_2307_04339_amd import ops
    x, _ = rand((n, hw, hw, c), dtype, 41)
    w, _ = rand((k, 3, 3, c), dtype, 42, -0.2, 0.2)
    rng = np.random.default_rng(43)
    bn = f32_dev(np.stack([rng.uniform(0.8, 1.2, k), rng.uniform(-0.1, 0.1, k), rng.uniform(-0.1, 0.1, k), rng.uniform(0.8, 1.2, k)]))
    y = empty((n, hw, hw, k), dtype)
    op = ops.conv2d(x, w, y, stride=1, pad=1, bias=None, bn=bn, residual=None, act="none", tile=8)
    assert op.info.path == L.PATH_RESIDENT
    got = []
    for block in (64, 128, 256):
        y.fill_(float("nan"))
        op.launch(0, op.T, op.T, block)
        torch.cuda.synchronize()
        got.append(bits(y))
    assert got[0] == got[1] == got[2]


@pytest.mark.parametrize("act", ["relu", "relu6", "gelu"])
def test_resident_conv_with_an_activation_in_every_block(act):
    from paper_2307_04339_amd import _lib as L
    from paper_2307_04339_amd import ops
    n, hw, c, k = 16, 56, 64, 64
    x, _ = rand((n, hw, hw, c), "f16", 44)
    w, _ = rand((k, 3, 3, c), "f16", 45, -0.2, 0.2)
    rng = np.random.default_rng(46)
    bn = f32_dev(np.stack([rng.uniform(0.8, 1.2, k), rng.uniform(-0.1, 0.1, k), rng.uniform(-0.1, 0.1, k), rng.uniform(0.8, 1.2, k)]))
    y = empty((n, hw, hw, k), "f16")
    op = ops.conv2d(x, w, y, stride=1, pad=1, bias=None, bn=bn, residual=None, act=act, tile=8)
    assert op.info.path == L.PATH_RESIDENT
    got = []
    for block in (64, 128, 256):
        y.fill_(float("nan"))
        op.launch(0, op.T, op.T, block)
        torch.cuda.synchronize()
        got.append(bits(y))
    assert got[0] == got[1] == got[2]
