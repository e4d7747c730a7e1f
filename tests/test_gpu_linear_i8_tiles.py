"""The 8-bit product's tiles of 128 rows where K is cut: sums of two and three chunks of 1,024, one net and ragged ones."""
import numpy as np
import pytest
import torch

from gpu_common import lib, need_gpu
from test_gpu_linear_i8 import check
from test_gpu_route import experts

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16], ids=["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,k,E,K,N,drop,act", [
    (2503, 2, 13, 1248, 517, 0.0, "tanh"), (2503, 2, 13, 2576, 517, 0.2, None), (4999, 1, 1, 2064, 600, 0.0, "tanh"),
    (1999, 1, 1, 1040, 900, 0.0, None), (3000, 2, 3, 3088, 390, 0.1, "tanh")])
def test_cut_sums(dtype, T, k, E, K, N, drop, act):
    dpc = lib()
    assert dpc.dp_linear_i8_work_bytes(T * k, K, N, E) == 0  # not the wide tiles
    r = np.random.default_rng(T + K)
    start = None
    if E > 1:
        start = dpc.dp_route_plan(torch.from_numpy(experts(T, T, k, E, drop)).cuda(), E)[0].cpu().numpy()
    xq, wq = (r.integers(-128, 128, s).astype(np.int8) for s in ((T * k, K), (E, N, K)))
    sx, sw = r.random(T * k).astype(np.float32), r.random((E, N)).astype(np.float32) / (64 * K)
    if start is not None:
        sx[start[-1]:] = np.nan
    check(dpc, xq, sx, wq, sw, r.normal(0, 0.1, (E, N)).astype(np.float32), start, act, dtype)


@pytest.mark.parametrize("K", [2064, 3088])
def test_sums_are_exact_at_their_largest(K):
    """Every product at its largest magnitude, and one odd unit, through tiles of 128 rows."""
    dpc = lib()
    rows, N = 4999, 520
    xq, wq = np.full((rows, K), -128, np.int8), np.full((1, N, K), -128, np.int8)
    xq[1::3], wq[0, 1::3] = 127, 127
    xq[2::3, ::2], wq[0, 2::3, 1::2] = 127, 127
    xq[5, 5] = 1
    wq[0, 3] = 0
    wq[0, 3, K - 1] = 1
    assert dpc.dp_linear_i8_work_bytes(rows, K, N, 1) == 0
    one = torch.ones(rows, device="cuda"), torch.ones(1, N, device="cuda")
    y = dpc.dp_linear_i8(torch.from_numpy(xq).cuda(), one[0], torch.from_numpy(wq).cuda(), one[1])
    exact = (xq.astype(np.float64) @ wq[0].astype(np.float64).T).astype(np.float32)  # sums below 2^53
    assert np.array_equal(y.cpu().numpy(), exact)
