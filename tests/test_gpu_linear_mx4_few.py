"""The 4-bit product of one and two rows, beside three and more, near the ends of f32's range and with scales of NaN."""
import numpy as np
import pytest
import torch

import mx4_common as M
from gpu_common import lib, need_gpu
from test_gpu_linear_mx4 import check, weights

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def product(xq, sx, wq, sw):
    return lib().dp_linear_mx4(*(torch.from_numpy(a).cuda() for a in (xq, sx, wq, sw)))


@pytest.mark.parametrize("ends", [(90, 165, 90, 165), (0, 60, 150, 200), (200, 250, 10, 50), (0, 20, 0, 250), (235, 255, 0, 20)])
@pytest.mark.parametrize("n", [1, 2])
def test_extreme_scales(ends, n):
    K, N = 320, 40
    r = np.random.default_rng(7)
    xq, wq = (r.integers(0, 256, s, dtype=np.uint8) for s in ((n, K // 2), (1, N, K // 2)))
    sx, sw = r.integers(ends[0], ends[1], (n, 16), dtype=np.uint8), r.integers(ends[2], ends[3], (1, N, 16), dtype=np.uint8)
    check(product(xq, sx, wq, sw), M.values(xq, sx), M.values(wq, sw)[0], np.zeros(N), None, torch.float32)


@pytest.mark.parametrize("n", [1, 2, 3, 70])
@pytest.mark.parametrize("ex", [127, 140, 200, 227, 246, 254])
def test_products_near_the_largest_number(n, ex):
    """Two elements a block, in two blocks: 6 x 6 2^(e + e'), up to 2^127, as the scales share the exponent."""
    K, N = 64, 9
    code = np.zeros((n, K), np.uint8)
    code[:, 0], code[:, 33] = 7, 2                 # 6 and 1
    wc = np.zeros((N, K), np.uint8)
    wc[:, 0], wc[:, 33] = 2, 9                     # 1 and -0.5
    sx, sw = np.zeros((n, 8), np.uint8), np.zeros((1, N, 8), np.uint8)
    sx[:, :2], sw[:, :, :2] = ex, 127 + 124 - (ex - 127)  # 2^124 together
    xq, wq = M.pack(code), M.pack(wc)[None]
    y = product(xq, sx, wq, sw).double().cpu().numpy()
    assert np.array_equal(y, np.full((n, N), 5.5 * 2.0 ** 124))


@pytest.mark.parametrize("n", [1, 2])
@pytest.mark.parametrize("top", [255 - 1, 192])
def test_a_block_that_sums_to_zero_under_large_scales(n, top):
    """Codes of zero, and codes whose products cancel, under scales that come to 2^128 and more: the block adds 0."""
    K, N = 128, 5
    code, wc = np.zeros((n, K), np.uint8), np.zeros((N, K), np.uint8)
    code[:, :2], wc[:, 0], wc[:, 1] = 7, 7, 15      # 6 x 6 - 6 x 6
    code[:, 40], wc[:, 41] = 7, 7                   # products of zeros
    code[:, 70], wc[:, 70] = 3, 4                   # 1.5 x 2
    sx, sw = np.full((n, 8), top, np.uint8), np.full((1, N, 8), 254, np.uint8)
    sx[:, 2], sw[:, :, 2] = 127, 127
    y = product(M.pack(code), sx, M.pack(wc)[None], sw)
    assert (y == 3).all()


@pytest.mark.parametrize("n", [1, 2])
def test_a_scale_of_nan(n):
    K, N = 576, 140
    r = np.random.default_rng(2)
    x = r.normal(size=(n, K))
    x[n - 1, 33] = np.inf
    xq, sx = lib().dp_quant_rows_mx4(torch.from_numpy(x).float().cuda())
    wq, sw, wv = weights(3, 1, N, K)
    sw[0, 20, 5] = 255
    y = lib().dp_linear_mx4(xq, sx, wq, sw).double().cpu().numpy()
    assert np.isnan(y[n - 1]).all() and np.isnan(y[:, 20]).all()
    ok = np.arange(N) != 20
    code, scale = M.quantise(x)
    check(y[: n - 1, ok], M.values(M.pack(code), scale)[: n - 1], wv[0][ok], np.zeros(N - 1), None, torch.float32)
