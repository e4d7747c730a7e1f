"""Routing of tokens to experts and back on the GPU: the plan against a stable sort, the moves bit for bit, the
weighted sums and gradients against 64 bits with elementwise bounds of their arithmetic, and central differences."""
import numpy as np
import pytest
import torch

from gpu_common import lib, need_gpu
from rows_common import IDS, ROWS, SUM_UNIT, TINY, UNIT, f64, offset_view, rnd, within, wtype

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def experts(seed, T, k, E, drop=0.2):
    r = np.random.default_rng(seed)
    e = r.integers(0, E, (T, k))
    bad = r.choice(np.array([-1, -2 ** 31, E, E + 7, 2 ** 31 - 1]), (T, k))
    return np.where(r.random((T, k)) < drop, bad, e).astype(np.int32)


def plan(expert, E):
    """The plan by a stable sort."""
    flat = expert.reshape(-1).astype(np.int64)
    key = np.where((flat >= 0) & (flat < E), flat, E)
    order = np.argsort(key, kind="stable")
    start = np.searchsorted(key[order], np.arange(E + 1))
    src = np.full(flat.size, -1)
    src[: start[E]] = order[: start[E]]
    pos = np.full(flat.size, -1)
    pos[src[: start[E]]] = np.arange(start[E])
    return start, src, pos.reshape(expert.shape)


@pytest.mark.parametrize("T,k,E,drop", [
    (0, 1, 3, 0.0), (1, 1, 1, 0.0), (1, 2, 8, 0.0), (33, 3, 5, 0.3), (511, 2, 1024, 0.1), (4096, 2, 8, 0.0),
    (4097, 2, 8, 0.2), (9001, 1, 2, 1.0), (16384, 2, 9, 0.1), (16385, 2, 9, 0.1), (4100, 1, 1024, 0.0), (14000, 2, 1000, 0.3), (32768, 1, 5, 0.0), (32769, 1, 5, 0.0), (20011, 3, 61, 0.2), (70001, 8, 7, 0.05), (3000, 5, 1023, 0.2),
    (700001, 1, 3, 0.1)])
def test_plan(T, k, E, drop):
    dpc = lib()
    e = experts(T + E, T, k, E, drop)
    start, src, pos = dpc.dp_route_plan(torch.from_numpy(e).cuda(), E)
    rs, rr, rp = plan(e, E)
    assert np.array_equal(start.cpu().numpy(), rs)
    assert np.array_equal(src.cpu().numpy(), rr)
    assert np.array_equal(pos.cpu().numpy(), rp)


def test_plan_of_one_expert_is_the_identity():
    dpc = lib()
    e = torch.full((10000, 2), 4, dtype=torch.int32, device="cuda")
    start, src, pos = dpc.dp_route_plan(e, 6)
    assert start.tolist() == [0, 0, 0, 0, 0, 20000, 20000]
    assert torch.equal(src, torch.arange(20000, dtype=torch.int32, device="cuda"))
    assert torch.equal(pos.reshape(-1), src)


SHAPES = [(1, 1, 1, 1, 0.0), (1, 2, 8, 240, 0.0), (37, 3, 5, 17, 0.3), (200, 2, 3, 1600, 0.1), (64, 4, 9, 1003, 0.2),
          (5, 1, 4, 5000, 0.5), (50, 2, 2, 130, 1.0), (0, 2, 3, 16, 0.0), (300, 1, 4, 4, 0.0)]


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,k,E,H,drop", SHAPES)
@pytest.mark.parametrize("offset", [0, 1])
def test_moves_and_gradients(dtype, T, k, E, H, drop, offset):
    """gather bit for bit; combine and its gradient within (k + 1) or (H + 1) roundings of the sums' type on the
    sum of magnitudes, plus one rounding to the row type.  NaN in the rows that no pair points to is not read."""
    dpc = lib()
    e = experts(7 * T + H, T, k, E, drop)
    start, src, pos = dpc.dp_route_plan(torch.from_numpy(e).cuda(), E)
    rs, rr, rp = plan(e, E)
    kept = int(rs[E])
    (x, xr), (z, zr), (dy, dyr) = (rnd(s, n, H, dtype=dtype) for s, n in ((1, T), (2, T * k), (3, T)))
    w, wr = rnd(4, T, k, dtype=wtype(dtype))
    if kept < T * k:
        z[kept:] = float("nan")
        zr[kept:] = 0.0
    if offset:
        x, z, dy = offset_view(x), offset_view(z), offset_view(dy)
    u, a = UNIT[dtype], SUM_UNIT[dtype]
    xs = dpc.dp_route_gather(x, src, pos)
    ref = np.zeros((T * k, H))
    ref[:kept] = xr[rr[:kept] // k]
    assert np.array_equal(f64(xs), ref)
    for weights, wv in ((w, wr), (None, np.ones((T, k)))):
        terms = np.where(rp >= 0, wv, 0.0)[:, :, None] * zr[np.maximum(rp, 0)] if T else np.zeros((0, k, H))
        y = dpc.dp_route_combine(z, pos, weights)
        yr = terms.sum(1)
        mag = np.abs(terms).sum(1)
        within(y, yr, (u + a) * np.abs(yr) + (k + 1) * a * (1 + u) * mag + TINY[dtype], "combine")
        dz, dw = dpc.dp_route_combine_grad(z, src, pos, weights, dy)
        dzr = np.zeros((T * k, H))
        dzr[:kept] = wv.reshape(-1)[rr[:kept], None] * dyr[rr[:kept] // k]
        within(dz, dzr, (u + 2 * a) * np.abs(dzr) + TINY[dtype], "dz")
        prod = np.where(rp >= 0, 1.0, 0.0)[:, :, None] * zr[np.maximum(rp, 0)] * dyr[:, None] if T else terms
        within(dw, prod.sum(2), (H + 1) * a * np.abs(prod).sum(2), "dw")
        alone, none = dpc.dp_route_combine_grad(None, src, pos, weights, dy, want=("dz",))
        assert none is None and torch.equal(alone, dz)


def test_gather_backward_is_combine_of_ones():
    """<gather(x), c> = <x, combine(c)>: the two are transposes of one another."""
    dpc = lib()
    e = torch.from_numpy(experts(5, 90, 3, 4, 0.3)).cuda()
    start, src, pos = dpc.dp_route_plan(e, 4)
    (x, xr), (c, cr) = rnd(1, 90, 33), rnd(2, 270, 33)
    lhs = (f64(dpc.dp_route_gather(x, src, pos)) * cr).sum()
    rhs = (xr * f64(dpc.dp_route_combine(c, pos))).sum()
    assert abs(lhs - rhs) <= 1e-12 * np.abs(cr).sum()


def test_gradient_against_differences():
    """d/dh of <dy, combine(z + h dz', w + h dw')> by central differences (the map is bilinear: only rounding,
    about 1e-16 |terms| / h, is left)."""
    dpc = lib()
    T, k, H = 40, 2, 50
    e = torch.from_numpy(experts(6, T, k, 5, 0.2)).cuda()
    start, src, pos = dpc.dp_route_plan(e, 5)
    (z, _), (w, _), (dy, _), (zd, zdr), (wd, wdr) = (rnd(s, *sh) for s, sh in (
        (1, (T * k, H)), (2, (T, k)), (3, (T, H)), (4, (T * k, H)), (5, (T, k))))
    dz, dw = dpc.dp_route_combine_grad(z, src, pos, w, dy)
    h = 1e-4
    loss = lambda s: float((dpc.dp_route_combine(z + s * zd, pos, w + s * wd) * dy).sum())  # noqa: E731
    num = (loss(h) - loss(-h)) / (2 * h)
    ana = (f64(dz) * zdr).sum() + (f64(dw) * wdr).sum()
    assert abs(num - ana) <= 1e-8 * (np.abs(f64(dz) * zdr).sum() + np.abs(f64(dw) * wdr).sum())


def test_other_stream_and_graph():
    """The calls run on the current stream, allocate nothing when given outputs, and replay as a graph."""
    dpc = lib()
    e = torch.from_numpy(experts(8, 6000, 2, 7, 0.1)).cuda()
    x, _ = rnd(1, 6000, 48, dtype=torch.float32)
    w = torch.rand(6000, 2, device="cuda")
    outs = dpc.dp_route_plan(e, 7)
    work = torch.empty(dpc.dp_route_work_bytes(6000, 2, 7), dtype=torch.uint8, device="cuda")
    xs, y = torch.empty(12000, 48, device="cuda"), torch.empty(6000, 48, device="cuda")

    def step():
        dpc.dp_route_plan(e, 7, out=outs, work=work)
        dpc.dp_route_gather(x, outs[1], outs[2], out=xs)
        dpc.dp_route_combine(xs, outs[2], w, out=y)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    first = y.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    x.mul_(2.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, 2.0 * first)


def test_refusals():
    dpc = lib()
    e = torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    start, src, pos = dpc.dp_route_plan(e, 3)
    x = torch.zeros(4, 8, device="cuda")
    with pytest.raises(TypeError):
        dpc.dp_route_plan(e.long(), 3)
    with pytest.raises(ValueError):
        dpc.dp_route_plan(e.reshape(-1), 3)
    with pytest.raises(ValueError):
        dpc.dp_route_plan(e, 0)
    with pytest.raises(ValueError):
        dpc.dp_route_plan(e, 1025)
    with pytest.raises(ValueError):
        dpc.dp_route_gather(x[:3], src, pos)
    with pytest.raises(ValueError):
        dpc.dp_route_gather(x, src[:7], pos)
    with pytest.raises(ValueError):
        dpc.dp_route_gather(torch.zeros(8, 4, device="cuda").t(), src, pos)
    with pytest.raises(TypeError):
        dpc.dp_route_gather(x.int(), src, pos)
    with pytest.raises(TypeError):
        dpc.dp_route_gather(x.cpu(), src, pos)
    with pytest.raises(ValueError):
        dpc.dp_route_combine(x, pos)
    z = torch.zeros(8, 8, device="cuda")
    with pytest.raises(TypeError):
        dpc.dp_route_combine(z, pos, torch.zeros(4, 2, dtype=torch.float64, device="cuda"))
    with pytest.raises(ValueError):
        dpc.dp_route_combine_grad(z, src, pos, None, x, want=("dw",))
    with pytest.raises(dpc.DPError) as err:
        dpc.dp_route_plan(torch.zeros(90000, 2, dtype=torch.int32, device="cuda"), 3,
                          work=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert err.value.code == dpc.DP_ERR_SHAPE
