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


# (T, H): whole rows to 2048, 4096 and 8192, a warp a row (16 bits), and rows under aligned words
@pytest.mark.parametrize("row", [0, 3000])
@pytest.mark.parametrize("dtype,T,H", [
    (torch.float32, 6000, 1600), (torch.float32, 5400, 2560), (torch.bfloat16, 6001, 1600), (torch.bfloat16, 6000, 2048),
    (torch.bfloat16, 5700, 4096), (torch.bfloat16, 5500, 6000), (torch.float64, 5300, 1024), (torch.bfloat16, 20001, 512), (torch.float16, 20001, 501),
    (torch.float16, 30003, 1003), (torch.float32, 30003, 1003)])
def test_norms(dtype, T, H, row):
    dpc = lib()
    g = torch.Generator("cuda").manual_seed(T + H)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    wd = torch.float64 if dtype == torch.float64 else torch.float32
    r, f, gate, dr2, du = (rn(T, H).to(dtype) for _ in range(5))
    a, w1, w2, b1, b2 = (rn(H).to(wd) for _ in range(5))

    def rows_left(got, good):
        lost = torch.isnan(got).view(T, -1)
        assert torch.equal(got.view(T, -1)[~lost], good.view(T, -1)[~lost])
        assert not lost[:max(row - 152 * 8, 0)].any() and lost[-1].all()  # a block may take the row before beside its first
        assert torch.equal(lost.any(1), lost.all(1))
        if row == 0:
            assert lost.all()

    for kind in ("rms", "layer"):
        kw = dict(b1=b1, b2=b2, gate=gate, kind=kind) if kind == "layer" else dict(gate=gate, kind=kind)
        forward = lambda: dpc.dp_norm_gate_fwd(r, f, a, w1, w2, **kw)  # noqa: E731
        good = forward()
        got, count = given_up(dpc, row, forward)
        assert count > 0
        rows_left(got[0], good[0])
        rows_left(got[1], good[1])
        rows_left(got[2][:, 3], good[2][:, 3])
        assert torch.equal(torch.isnan(got[2][:, 1]), torch.isnan(got[2][:, 3]))
        assert all(torch.equal(x, y) for x, y in zip(forward(), good))

        if H == 501:
            continue  # the backward takes these by elements: no waits
        backward = lambda: dpc.dp_norm_gate_grad(good[0], f, a, w1, w2, good[2], dr2, du, **kw)  # noqa: E731
        ref = backward()
        got, count = given_up(dpc, row, backward)
        assert count > 0
        for n in ("dr", "df", "dgate"):
            rows_left(got[n], ref[n])
        for n in ("da", "dw1", "dw2", "db1", "db2"):
            assert got[n] is None or torch.isnan(got[n]).all(), n
        again = backward()
        assert all(x is None or torch.equal(x, again[n]) for n, x in ref.items())
    assert dpc.dp_tc_wait_timeouts() == 0


def test_rows_past_the_last_are_no_rows():
    dpc = lib()
    x, v = torch.randn(300, 1600, device="cuda"), torch.ones(1600, device="cuda")
    good = dpc.dp_norm_gate_fwd(x, x, v, v, v)
    got, count = given_up(dpc, 300, lambda: dpc.dp_norm_gate_fwd(x, x, v, v, v))
    assert count == 0 and all(torch.equal(a, b) for a, b in zip(good, got))
