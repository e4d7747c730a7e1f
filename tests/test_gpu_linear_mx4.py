"""Rows to microscaled 4-bit floating point on the GPU bit for bit, and their product with 4-bit weights against 64 bits
on the values that codes and scales stand for."""
import numpy as np
import pytest
import torch

import mx4_common as M
from gpu_common import lib, need_gpu
from rows_common import IDS, ROWS, TINY, UNIT, f64, offset_view, within
from test_gpu_route import experts, plan

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def rows(seed, n, K, dtype):
    """Rows of very different sizes, and within them blocks of zeros, ties between codes and the ends of the range."""
    r = np.random.default_rng(seed)
    x = r.normal(size=(n, K)) * np.exp(r.normal(size=(n, 1)) * 3)
    x[:, ::7] *= 8
    if n > 6 and K >= 64:
        x[1, :32] = 0.0
        ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.5, 6.5, 7.5, 4.0, -0.25, -0.75, -5.0, -0.1, -0.0])
        x[2, :32] = np.tile(ties, 2)
        x[3, :32] = np.tile(ties, 2) * 2.0 ** -10
        x[4] = 1e-7 if dtype != torch.float16 else 6e-8
        x[5] = float(torch.finfo(dtype).max) if dtype != torch.float64 else 3e38
        x[6, 32:64] = 2.0 ** -149 if dtype in (torch.float64, torch.float32) else float(torch.finfo(dtype).tiny)
        x[6, :32] = -x[6, 32:64]
    t = torch.from_numpy(x).to(dtype).cuda()
    return t, f64(t)


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("n,K", [(1, 1), (1, 240), (7, 32), (9, 64), (8, 65), (9, 255), (9, 256), (9, 257), (40, 1003), (33, 1600), (3, 65536), (0, 40), (2000, 96)])
@pytest.mark.parametrize("offset", [0, 1])
def test_quantise(dtype, n, K, offset):
    dpc = lib()
    x, xr = rows(n + K, n, K, dtype)
    xq, sx = dpc.dp_quant_rows_mx4(offset_view(x) if offset else x)
    code, scale = M.quantise(xr)
    assert np.array_equal(sx.cpu().numpy(), scale)
    assert np.array_equal(xq.cpu().numpy(), M.pack(code))


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
def test_quantise_infinities_and_nan(dtype):
    dpc = lib()
    x, _ = rows(3, 12, 300, dtype)
    x[7, 40], x[8, 290], x[9, 0], x[9, 31] = float("nan"), float("inf"), -float("inf"), float("nan")
    xq, sx = dpc.dp_quant_rows_mx4(x)
    code, scale = M.quantise(f64(x))
    assert np.array_equal(sx.cpu().numpy(), scale) and np.array_equal(xq.cpu().numpy(), M.pack(code))
    assert scale[7, 1] == scale[8, 9] == scale[9, 0] == 255 and (scale == 255).sum() == 3


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,k,E,K", [(1, 2, 8, 240), (37, 3, 5, 70), (300, 2, 4, 1003), (20, 1, 3, 16)])
def test_quantise_to_sorted_places(dtype, T, k, E, K):
    dpc = lib()
    x, xr = rows(T, T, K, dtype)
    e = experts(T, T, k, E, 0.2)
    rs, rr, _ = plan(e, E)
    _, src, pos = dpc.dp_route_plan(torch.from_numpy(e).cuda(), E)
    ldq, lds = (K + 63) // 64 * 64, (K + 255) // 256 * 8
    out = torch.full((T * k, ldq // 2), 77, dtype=torch.uint8, device="cuda"), torch.full((T * k, lds), 77, dtype=torch.uint8, device="cuda")
    xq, sx = dpc.dp_quant_rows_mx4(x, src, pos, out=out)
    code, scale = M.quantise(xr)
    want_q, want_s = np.zeros((T * k, ldq // 2), np.uint8), np.zeros((T * k, lds), np.uint8)
    kept = int(rs[E])
    want_q[:kept], want_s[:kept] = M.pack(code)[rr[:kept] // k], scale[rr[:kept] // k]
    assert np.array_equal(xq.cpu().numpy(), want_q) and np.array_equal(sx.cpu().numpy(), want_s)


def weights(seed, E, N, K):
    """(wq, sw) on the GPU and the values [E][N][ldq]; padded columns hold zero codes."""
    r = np.random.default_rng(seed)
    code, scale = M.quantise((r.normal(size=(E * N, K)) * np.exp(r.normal(size=(E * N, 1)))))
    q, s = M.pack(code).reshape(E, N, -1), scale.reshape(E, N, -1)
    return torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda(), M.values(q, s)


def check(y, x, w, bias, act, dtype, what=""):
    """x [n][K], w [N][K] values.  Products are exact; K additions of the sum, each of which may lose a unit in the last
    place (2^-23) of a partial sum that the magnitudes bound; the bias's addition; tanh's own 2 ulp, its derivative at
    most 1; one rounding to the row type (f64 rows hold f32 values)."""
    ref = x @ w.T + bias
    mag = np.abs(x) @ np.abs(w).T + np.abs(bias)
    b = mag * (x.shape[1] + 4) * 2.0 ** -23
    if act:
        ref = np.tanh(ref)
        b = np.minimum(b, 2.0) + 4 * 2.0 ** -24
    unit = max(UNIT[dtype], 2.0 ** -24)
    # what lies beyond the row type's largest value rounds to an infinity: both count as that value
    top = float(torch.finfo(dtype).max)
    y, ref = np.clip(y if isinstance(y, np.ndarray) else f64(y), -top, top), np.clip(ref, -top, top)
    within(y, ref, b + (np.abs(ref) + b) * unit + TINY[dtype], what)


PRODUCTS = [(1, 64, 1, 1), (1, 1600, 100, 1), (3, 240, 33, 1), (16, 1003, 70, 1), (17, 64, 5, 1), (17, 1237, 517, 1), (64, 256, 128, 1), (65, 512, 129, 1), (130, 320, 260, 1),
            (300, 96, 17, 1), (500, 1600, 240, 1), (1000, 2048, 300, 1), (40, 4096, 64, 1), (2000, 64, 64, 1),
            # tiles of 128 and of 192 rows
            (12000, 320, 260, 1), (30000, 64, 300, 1), (6000, 1088, 2100, 1), (2, 512, 33, 1), (2, 4096, 2100, 1), (4, 1600, 300, 1)]


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("n,K,N,E", PRODUCTS)
@pytest.mark.parametrize("act", [None, "tanh"])
def test_product(dtype, n, K, N, E, act):
    dpc = lib()
    r = np.random.default_rng(n + N)
    code, scale = M.quantise(r.normal(size=(n, K)) * np.exp(2 * r.normal(size=(n, 1))) / K ** 0.5)
    xq, sx = torch.from_numpy(M.pack(code)).cuda(), torch.from_numpy(scale).cuda()
    wq, sw, wv = weights(K, E, N, K)
    bias = torch.from_numpy(r.normal(size=(E, N))).float().cuda()
    y = dpc.dp_linear_mx4(xq, sx, wq, sw, bias=bias, act=act, dtype=dtype)
    assert y.dtype == dtype
    xv = M.values(M.pack(code), scale)
    check(y, xv, wv[0], f64(bias)[0], act, dtype)
    if act is None:
        check(dpc.dp_linear_mx4(xq, sx, wq, sw, dtype=dtype), xv, wv[0], np.zeros(N), act, dtype, "no bias")


@pytest.mark.parametrize("scales", ["far apart", "lowest", "highest"])
@pytest.mark.parametrize("n", [5, 200])
def test_product_of_extreme_scales(scales, n):
    """Scales far apart within a row, and near the ends of f32's range."""
    dpc = lib()
    K, N = 320, 40
    r = np.random.default_rng(7)
    xq, wq = (r.integers(0, 256, s, dtype=np.uint8) for s in ((n, K // 2), (1, N, K // 2)))
    lo, hi = {"far apart": (90, 165), "lowest": (0, 60), "highest": (200, 250)}[scales]
    sx = r.integers(lo, hi, (n, 16), dtype=np.uint8)
    sw = r.integers(*{"far apart": (90, 165), "lowest": (150, 200), "highest": (10, 50)}[scales], (1, N, 16), dtype=np.uint8)
    y = dpc.dp_linear_mx4(*(torch.from_numpy(a).cuda() for a in (xq, sx, wq, sw)))
    check(y, M.values(xq, sx), M.values(wq, sw)[0], np.zeros(N), None, torch.float32)


@pytest.mark.parametrize("n", [9, 300])
def test_a_scale_of_nan_spoils_its_row_or_channel_only(n):
    dpc = lib()
    K, N = 576, 140
    r = np.random.default_rng(2)
    x = r.normal(size=(n, K))
    x[4, 33], x[7, 570] = np.inf, np.nan
    xq, sx = dpc.dp_quant_rows_mx4(torch.from_numpy(x).float().cuda())
    wq, sw, wv = weights(3, 1, N, K)
    sw[0, 20, 5] = 255
    y = f64(dpc.dp_linear_mx4(xq, sx, wq, sw))
    bad_r, bad_c = np.zeros(n, bool), np.zeros(N, bool)
    bad_r[[4, 7]], bad_c[20] = True, True
    assert np.isnan(y[bad_r]).all() and np.isnan(y[:, bad_c]).all()
    code, scale = M.quantise(x)
    check(y[np.ix_(~bad_r, ~bad_c)], M.values(M.pack(code), scale)[~bad_r], wv[0][~bad_c], np.zeros((~bad_c).sum()), None, torch.float32)


EXPERTS = [(1, 2, 8, 240, 100), (6, 2, 3, 64, 9), (40, 2, 5, 96, 130), (400, 2, 13, 1237, 150), (300, 3, 61, 70, 31), (900, 1, 4, 320, 240), (700, 2, 2, 512, 64), (50, 1, 1024, 64, 7), (9000, 2, 5, 96, 800), (300, 2, 1, 96, 130), (500, 1, 1, 1100, 200)]


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,k,E,K,N", EXPERTS)
@pytest.mark.parametrize("drop", [0.0, 0.2])
def test_experts(dtype, T, k, E, K, N, drop):
    """Ragged experts, some without rows; rows past the kept ones are zero rows."""
    dpc = lib()
    e = experts(T + E, T, k, E, drop)
    rs, rr, _ = plan(e, E)
    start, src, pos = dpc.dp_route_plan(torch.from_numpy(e).cuda(), E)
    x, xr = rows(T + 1, T, K, torch.float32)
    x = (x / x.abs().amax(1, keepdim=True).clamp(min=1e-30)).to(dtype)
    xq, sx = dpc.dp_quant_rows_mx4(x, src, pos)
    wq, sw, wv = weights(K, E, N, K)
    r = np.random.default_rng(1)
    bias = torch.from_numpy(r.normal(size=(E, N))).float().cuda()
    out = torch.full((T * k, N), float("nan"), dtype=dtype, device="cuda")
    y = dpc.dp_linear_mx4(xq, sx, wq, sw, bias=bias, start=start, act="tanh", dtype=dtype, out=out)
    xv = M.values(xq.cpu().numpy(), sx.cpu().numpy())
    for n in range(E):
        check(y[rs[n]: rs[n + 1]], xv[rs[n]: rs[n + 1]], wv[n], f64(bias)[n], "tanh", dtype, f"expert {n}")
    assert not y[rs[E]:].any()


@pytest.mark.parametrize("T,E,N", [(1, 1, 5), (5, 3, 200), (700, 4, 130), (3000, 64, 7)])
def test_every_pair_dropped(T, E, N):
    """No expert has a row: every row of the result is zero."""
    dpc = lib()
    start, src, pos = dpc.dp_route_plan(torch.full((T, 2), -1, dtype=torch.int32, device="cuda"), E)
    x, _ = rows(T, T, 320, torch.float32)
    xq, sx = dpc.dp_quant_rows_mx4(x, src, pos)
    assert not xq.any()
    wq, sw, _ = weights(N, E, N, 320)
    out = torch.full((T * 2, N), float("nan"), device="cuda")
    dpc.dp_linear_mx4(xq, sx, wq, sw, bias=torch.ones(E, N, device="cuda"), start=start, act="tanh", out=out)
    assert (out == 0).all()


def test_rows_behind_the_output_stay(dtype=torch.float32):
    """Nothing is written past the last row or channel."""
    dpc = lib()
    n, K, N = 150, 128, 131
    r = np.random.default_rng(5)
    code, scale = M.quantise(r.normal(size=(n, K)))
    wq, sw, wv = weights(4, 1, N, K)
    buf = torch.full((n * N + 4096,), 7.0, device="cuda")
    y = buf[2048: 2048 + n * N].view(n, N)
    dpc.dp_linear_mx4(torch.from_numpy(M.pack(code)).cuda(), torch.from_numpy(scale).cuda(), wq, sw, out=y)
    assert (buf[:2048] == 7).all() and (buf[2048 + n * N:] == 7).all()
    check(y, M.values(M.pack(code), scale), wv[0], np.zeros(N), None, dtype)


def test_graph_and_repeats():
    """Captured with the quantiser and replayed on new rows; the same inputs give the same bits."""
    dpc = lib()
    n, K, N = 600, 800, 200
    wq, sw, _ = weights(6, 1, N, K)
    x, _ = rows(1, n, K, torch.bfloat16)
    x = torch.nan_to_num(x).clamp(-100, 100)
    xq, sx = dpc.dp_quant_rows_mx4(x)
    want = dpc.dp_linear_mx4(xq, sx, wq, sw, act="tanh", dtype=torch.bfloat16)
    for _ in range(3):
        assert torch.equal(dpc.dp_linear_mx4(xq, sx, wq, sw, act="tanh", dtype=torch.bfloat16), want)
    q, s, y, xin = torch.empty_like(xq), torch.empty_like(sx), torch.empty_like(want), torch.zeros_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dpc.dp_quant_rows_mx4(xin, out=(q, s))
        dpc.dp_linear_mx4(q, s, wq, sw, act="tanh", dtype=torch.bfloat16, out=y)
    xin.copy_(x)
    graph.replay()
    assert torch.equal(y, want)


@pytest.mark.parametrize("stage", [0, 1, 2, 5, 23])
@pytest.mark.parametrize("n,K,N", [(60, 64, 200), (700, 2304, 1000), (12000, 320, 260), (9000, 2048, 1300)])
def test_waits_that_give_up(n, K, N, stage):
    """Bounded waits that give up, as a test hook makes them: the outputs they leave are NaN, all others right, the count
    says so, and the next call is sound."""
    dpc = lib()
    assert dpc.dp_tc_wait_timeouts() == 0
    g = torch.Generator("cuda").manual_seed(n)
    u8 = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, dtype=torch.uint8, device="cuda")  # noqa: E731
    lds = (K + 255) // 256 * 8
    args = u8(0, 256, n, K // 2), u8(120, 130, n, lds), u8(0, 256, 1, N, K // 2), u8(120, 130, 1, N, lds)
    good = dpc.dp_linear_mx4(*args)
    assert not torch.isnan(good).any()
    try:
        dpc.dp_give_up_at(stage)
        got = dpc.dp_linear_mx4(*args)
    finally:
        dpc.dp_give_up_at(-1)
    count = dpc.dp_tc_wait_timeouts()
    lost = torch.isnan(got)
    assert torch.equal(got[~lost], good[~lost])
    assert bool(lost.any()) == (count > 0) == (stage < -(-K // 256) or count > 0)
    if stage == 0:
        assert lost.all()
    assert torch.equal(dpc.dp_linear_mx4(*args), good) and dpc.dp_tc_wait_timeouts() == 0


def test_products_on_two_streams_at_once():
    dpc = lib()
    cases = []
    for n, K, N in ((3000, 1088, 700), (500, 2304, 1500)):
        r = np.random.default_rng(n)
        code, scale = M.quantise(r.normal(size=(n, K)))
        args = torch.from_numpy(M.pack(code)).cuda(), torch.from_numpy(scale).cuda(), *weights(n, 1, N, K)[:2]
        cases.append((args, dpc.dp_linear_mx4(*args), []))
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, (args, _, got) in zip(streams, cases):
            with torch.cuda.stream(st):
                got.append(dpc.dp_linear_mx4(*args))
    torch.cuda.synchronize()
    for _, want, got in cases:
        assert all(torch.equal(y, want) for y in got)
