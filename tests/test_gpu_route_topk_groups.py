"""Groups whose scores are sums that cancel or pass f32's range: the groups kept against extended precision, exactly."""
import numpy as np
import pytest
import torch

from gpu_common import lib, need_gpu
from test_gpu_route_topk import reference

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()



@pytest.mark.parametrize("dtype", [torch.float64, torch.float32, torch.bfloat16], ids=["f64", "f32", "bf16"])
@pytest.mark.parametrize("per,k", [(4, 2), (16, 9), (48, 40)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_sums_past_the_types_range(dtype, per, k, kind):
    """A group masked with the type's lowest value still stands above one masked with -inf, though the sum of two is
    -inf in the type; sums that pass the upper end are told apart."""
    dpc = lib()
    wd = torch.float64 if dtype == torch.float64 else torch.float32
    low, inf = float(torch.finfo(wd).min), float("inf")
    x = torch.linspace(2.0, -2.0, 3 * per)[None].expand(5, -1).to(dtype).contiguous().cuda()
    b = torch.full((3, per), -inf, dtype=wd, device="cuda")
    b[1], b[2] = low, low
    e, w = dpc.dp_route_topk(x, k, bias=b.view(-1), score=kind, ngroup=3, keep_groups=1, renorm=False)
    assert ((e >= per) & (e < 2 * per)).all()
    assert torch.equal(e, torch.arange(per, per + k, device="cuda", dtype=torch.int32).expand(5, -1))
    b[0] = -low / 2
    b[1, :2], b[2, :2] = -low * 0.75, -low * 0.875
    e, _ = dpc.dp_route_topk(x, k, bias=b.view(-1), score=kind, ngroup=3, keep_groups=1)
    assert (e[:, :2] >= 2 * per).all()


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,G,keep,k", [(4, 2, 1, 2), (32, 2, 1, 2), (32, 8, 4, 6), (32, 2, 1, 9), (96, 6, 2, 20), (600, 12, 5, 8), (600, 12, 5, 40)])
@pytest.mark.parametrize("big", [300.0, 20000.0])
def test_sums_of_two_that_cancel(kind, E, G, keep, k, big):
    """The two best of every group have biases of +big and -big + 0.5: their roundings are those of big, the sum is not."""
    dpc = lib()
    T, per = 4000, E // G
    r = np.random.default_rng(E + k)
    x = r.normal(size=(T, E)).astype(np.float32)
    b = np.full((G, per), -2 * big, np.float32)
    for g in range(G):
        at = r.permutation(per)
        b[g, at[0]], b[g, at[1]] = big, -big + 0.5
    b = b.reshape(-1)
    e, _ = dpc.dp_route_topk(torch.from_numpy(x).cuda(), k, bias=torch.from_numpy(b).cuda(), score=kind, ngroup=G, keep_groups=keep)
    re, _ = reference(x.astype(np.float64), b.astype(np.float64), k, kind, G, keep, 2, True, 1.0)
    kept, rkept = (np.sort(v // per, 1) for v in (e.cpu().numpy(), re))
    assert np.array_equal(kept, rkept)
    assert np.array_equal(e.cpu().numpy(), re)
