"""Bounded waits that give up, as a test hook makes them: the outputs they leave are NaN, all others right, the count says
so, and the next call is sound.  Nothing hangs or faults: what is in flight is waited for."""
import pytest
import torch

from gpu_common import lib, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()
    assert lib().dp_tc_wait_timeouts() == 0
    yield
    lib().dp_give_up_at(-1)


def given_up(dpc, n, step):
    """step()'s outputs with the waits of stage (row) n given up, and how many were counted."""
    dpc.dp_give_up_at(n)
    out = step()
    dpc.dp_give_up_at(-1)
    return out, dpc.dp_tc_wait_timeouts()


@pytest.mark.parametrize("stage", [0, 1, 3, 4, 17, 40])
@pytest.mark.parametrize("rows,K,N", [(60, 64, 200), (2000, 1040, 900), (2100, 2064, 2100), (9000, 1024, 1024)])
def test_product(rows, K, N, stage):
    """Tiles of 64, of 128, and the wide ones, with the stages behind the given-up one on their way."""
    dpc = lib()
    g = torch.Generator("cuda").manual_seed(rows)
    xq, wq = (torch.randint(-127, 128, s, generator=g, dtype=torch.int8, device="cuda") for s in ((rows, K), (1, N, K)))
    sx, sw = torch.rand(rows, generator=g, device="cuda"), torch.rand(1, N, generator=g, device="cuda")
    good = dpc.dp_linear_i8(xq, sx, wq, sw)
    got, count = given_up(dpc, stage, lambda: dpc.dp_linear_i8(xq, sx, wq, sw))
    lost = torch.isnan(got)
    assert torch.equal(got[~lost], good[~lost])
    assert bool(lost.any()) == (count > 0) == (stage < -(-K // 64) or count > 0)
    if stage == 0:
        assert lost.all()
    assert torch.equal(dpc.dp_linear_i8(xq, sx, wq, sw), good) and dpc.dp_tc_wait_timeouts() == 0
