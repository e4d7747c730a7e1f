"""Rows as 8-bit integers and their product with 8-bit weights on the GPU: the integers bit for bit against the
definition in numpy, the product against exact integer sums with elementwise bounds of its f32 epilogue."""
import numpy as np
import pytest
import torch

from gpu_common import lib, need_gpu
from rows_common import IDS, ROWS, TINY, UNIT, f64, offset_view, rnd, within
from test_gpu_route import experts

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def quant(x):
    """The definition, in f32."""
    x = x.astype(np.float32)
    K = x.shape[1]
    q = np.zeros((x.shape[0], -(-K // 16) * 16), np.int8)
    s = np.zeros(x.shape[0], np.float32)
    for i, row in enumerate(x):
        if not np.all(np.isfinite(row)):
            s[i] = np.nan
            continue
        amax = np.abs(row).max()
        if amax >= np.float32(2.0 ** -100):
            q[i, :K] = np.rint(row * (np.float32(127) / amax))
            s[i] = amax / np.float32(127)
    return q, s


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,K", [(0, 5), (1, 1), (1, 16), (3, 17), (65, 240), (20, 1003), (9, 1600), (4, 9000), (2, 65536)])
@pytest.mark.parametrize("offset", [0, 1])
def test_rows_to_integers(dtype, T, K, offset):
    dpc = lib()
    x, _ = rnd(T + K, T, K, dtype=dtype, scale=3.0)
    if T >= 9:  # a zero row, tiny ones, halves (ties), infinities, NaN, and the type's largest value
        x[0] = 0
        x[1] *= 1e-30 if dtype != torch.float16 else 1e-6
        x[2] = (torch.arange(K, device="cuda") % 255 - 127).to(dtype) * 0.5
        x[2, 0] = 127
        x[3, K // 2] = float("inf")
        x[4, K - 1] = float("nan")
        x[5, 0] = torch.finfo(dtype).max if dtype != torch.float64 else 3e38
        x[6] = 1e-31 if dtype != torch.float16 else 0
    xr = x.double().cpu().numpy()
    if offset:
        x = offset_view(x)
    xq, sx = dpc.dp_quant_rows_i8(x)
    rq, rs = quant(xr)
    assert np.array_equal(xq.cpu().numpy(), rq)
    assert np.array_equal(sx.cpu().numpy(), rs, equal_nan=True)


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,k,E,K,drop", [(1, 1, 1, 16, 0.0), (1, 2, 8, 240, 0.0), (77, 3, 5, 133, 0.3), (20, 2, 3, 48, 1.0)])
def test_rows_to_integers_at_sorted_places(dtype, T, k, E, K, drop):
    """The fused form is the gather of the unfused one's rows."""
    dpc = lib()
    start, src, pos = dpc.dp_route_plan(torch.from_numpy(experts(T + K, T, k, E, drop)).cuda(), E)
    x, xr = rnd(3, T, K, dtype=dtype)
    xq, sx = dpc.dp_quant_rows_i8(x, src, pos)
    rq, rs = quant(xr)
    p = src.cpu().numpy()
    assert np.array_equal(xq.cpu().numpy(), np.where(p[:, None] >= 0, rq[np.maximum(p, 0) // k], 0))
    assert np.array_equal(sx.cpu().numpy(), np.where(p >= 0, rs[np.maximum(p, 0) // k], 0))


def product(xq, sx, wq, sw, bias, start, act):
    """Exact integer sums, the rest in f64; also the magnitude that the f32 roundings are relative to."""
    rows, (E, N, K) = xq.shape[0], wq.shape
    y, mag = np.zeros((rows, N)), np.zeros((rows, N))
    start = [0, rows] if start is None else start
    for e in range(E):
        r = slice(start[e], start[e + 1])
        dot = xq[r].astype(np.float64) @ wq[e].astype(np.float64).T  # exact: below 2^53
        v = dot * sx[r, None].astype(np.float64) * sw[e].astype(np.float64)
        y[r] = v + bias[e]
        mag[r] = np.abs(v) + np.abs(bias[e])
    return (np.tanh(y) if act else y), mag


def check(dpc, xq, sx, wq, sw, bias, start, act, dtype):
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    y = dpc.dp_linear_i8(dev(xq), dev(sx), dev(wq), dev(sw), None if bias is None else dev(bias),
                         None if start is None else dev(start.astype(np.int64)), act, dtype)
    ref, mag = product(xq, sx, wq, sw, np.zeros_like(sw) if bias is None else bias.astype(np.float64), start, act)
    if start is not None:
        assert not y[int(start[-1]):].any()
    # four f32 roundings (the integer, two products, the sum); tanh shrinks errors and adds its own, at most
    # 4 f32 units, or 2^-10 of the value where the result is rounded to bf16 anyway
    bound = 4 * U32 * mag + UNIT[dtype if dtype != torch.float64 else torch.float32] * np.abs(ref) + TINY[dtype]
    if act:
        bound += (2.0 ** -10 if dtype == torch.bfloat16 else 4 * U32) * np.abs(ref)
    within(y, ref, bound, "product")
    return y


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("rows,K,N", [
    (1, 16, 1), (1, 1600, 240), (2, 240, 2048), (7, 1248, 517), (9, 64, 33), (33, 2048, 129), (64, 80, 128),
    (100, 48, 300), (129, 1040, 257), (256, 256, 128), (300, 4112, 130), (513, 1600, 240), (1000, 96, 1000), (0, 32, 8)])
def test_one_net(dtype, rows, K, N):
    dpc = lib()
    r = np.random.default_rng(rows + K + N)
    xq, wq = (r.integers(-127, 128, s).astype(np.int8) for s in ((rows, K), (1, N, K)))
    sx, sw = r.random(rows).astype(np.float32) * 0.02, r.random((1, N)).astype(np.float32) / (64 * K ** 0.5)
    check(dpc, xq, sx, wq, sw, r.normal(0, 0.1, (1, N)).astype(np.float32), None, "tanh", dtype)
    check(dpc, xq, sx, wq, sw, None, None, None, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,k,E,K,N,drop", [
    (1, 2, 8, 1600, 240, 0.0), (40, 2, 61, 240, 130, 0.2), (500, 2, 3, 128, 64, 0.3), (700, 1, 5, 1104, 200, 0.0),
    (3000, 2, 13, 144, 517, 0.1), (64, 1, 1, 64, 96, 0.5), (90, 2, 4, 32, 40, 1.0), (5, 1, 1024, 48, 24, 0.0)])
def test_experts(dtype, T, k, E, K, N, drop):
    """Ragged experts, empty ones, rows past the kept ones (their sx is NaN here: zeros all the same)."""
    dpc = lib()
    r = np.random.default_rng(T + E + K)
    start, src, pos = dpc.dp_route_plan(torch.from_numpy(experts(T, T, k, E, drop)).cuda(), E)
    start = start.cpu().numpy()
    xq, wq = (r.integers(-128, 128, s).astype(np.int8) for s in ((T * k, K), (E, N, K)))
    sx, sw = r.random(T * k).astype(np.float32), r.random((E, N)).astype(np.float32) / (64 * K)
    sx[start[-1]:] = np.nan
    check(dpc, xq, sx, wq, sw, r.normal(0, 0.1, (E, N)).astype(np.float32), start, None, dtype)


@pytest.mark.parametrize("rows", [3, 300])
@pytest.mark.parametrize("K", [1024, 1040, 1600, 2064, 4112, 65536])
def test_sums_are_exact_at_their_largest(rows, K):
    """Every product at its largest magnitude, one sign or both, and one odd unit: the integer sum must not lose
    its last bit before its only rounding to f32 (rows of -128, and of 127 with a lone 1)."""
    dpc = lib()
    xq = np.full((rows, K), -128, np.int8)
    xq[1] = 127
    xq[2] = np.where(np.arange(K) % 2, 127, -127)
    xq[2, 5] = 1
    wq = np.full((1, 140, K), -128, np.int8)
    wq[0, 1] = 127
    wq[0, 2] = np.where(np.arange(K) % 2, 127, -127)
    wq[0, 3] = 0
    wq[0, 3, K - 1] = 1
    one = np.ones(rows, np.float32), np.ones((1, 140), np.float32)
    y = dpc.dp_linear_i8(*(torch.from_numpy(a).cuda() for a in (xq, one[0], wq, one[1])))
    exact = (xq.astype(np.int64) @ wq[0].astype(np.int64).T).astype(np.float32)
    assert np.array_equal(y.cpu().numpy(), exact)


def test_not_finite_rows_stay_in_their_rows():
    dpc = lib()
    x, _ = rnd(1, 200, 64, dtype=torch.float32)
    x[7, 3], x[150, 0] = float("nan"), float("-inf")
    w, _ = rnd(2, 128, 64, dtype=torch.float32)
    wq, sw = dpc.dp_quant_rows_i8(w)
    xq, sx = dpc.dp_quant_rows_i8(x)
    y = dpc.dp_linear_i8(xq, sx, wq.view(1, 128, 64), sw.view(1, 128), act="tanh")
    bad = torch.isnan(y)
    assert bad[7].all() and bad[150].all() and int(bad.sum()) == 256


def test_quantised_layer_is_near_the_layer():
    """A 1600 -> 240 layer in 8 bits: each factor is off by at most half a step, s_x / 2 and s_w / 2, so the sum
    is within sum_k (|x| s_w / 2 + |w| s_x / 2 + s_x s_w / 4)."""
    dpc = lib()
    (x, xr), (w, wr) = rnd(1, 300, 1600, dtype=torch.float32), rnd(2, 240, 1600, dtype=torch.float32, scale=0.025)
    xq, sx = dpc.dp_quant_rows_i8(x)
    wq, sw = dpc.dp_quant_rows_i8(w)
    y = dpc.dp_linear_i8(xq, sx, wq.view(1, 240, 1600), sw.view(1, 240))
    hx, hw = f64(sx)[:, None] * 0.5001, f64(sw)[None] * 0.5001
    bound = np.abs(xr).sum(1)[:, None] * hw + np.abs(wr).sum(1)[None] * hx + 1600 * hx * hw
    within(y, xr @ wr.T, bound, "layer")


def test_other_stream_and_graph():
    dpc = lib()
    x, _ = rnd(1, 500, 96, dtype=torch.bfloat16)
    w, _ = rnd(2, 200, 96, dtype=torch.float32)
    wq, sw = dpc.dp_quant_rows_i8(w)
    xq, sx = dpc.dp_quant_rows_i8(x)
    y = torch.empty(500, 200, dtype=torch.bfloat16, device="cuda")

    def step():
        dpc.dp_quant_rows_i8(x, out=(xq, sx))
        dpc.dp_linear_i8(xq, sx, wq.view(1, 200, 96), sw.view(1, 200), dtype=torch.bfloat16, out=y)

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
    x = torch.zeros(4, 32, device="cuda")
    xq, sx = dpc.dp_quant_rows_i8(x)
    wq, sw = torch.zeros(1, 8, 32, dtype=torch.int8, device="cuda"), torch.zeros(1, 8, device="cuda")
    start, src, pos = dpc.dp_route_plan(torch.zeros(4, 1, dtype=torch.int32, device="cuda"), 2)
    with pytest.raises(ValueError):
        dpc.dp_quant_rows_i8(x, src=src)
    with pytest.raises(ValueError):
        dpc.dp_quant_rows_i8(x[:3], src, pos)
    with pytest.raises(TypeError):
        dpc.dp_quant_rows_i8(x.int())
    with pytest.raises(dpc.DPError) as err:
        dpc.dp_quant_rows_i8(torch.zeros(1, 65537, device="cuda"))
    assert err.value.code == dpc.DP_ERR_UNSUPPORTED
    with pytest.raises(TypeError):
        dpc.dp_linear_i8(x, sx, wq, sw)
    with pytest.raises(ValueError):
        dpc.dp_linear_i8(xq, sx[:3], wq, sw)
    with pytest.raises(ValueError):
        dpc.dp_linear_i8(xq, sx, wq, sw, act="relu")
    with pytest.raises(TypeError):
        dpc.dp_linear_i8(xq, sx, wq, sw, dtype=torch.int32)
    with pytest.raises(ValueError):
        dpc.dp_linear_i8(xq, sx, wq, sw, start=start)
    with pytest.raises(dpc.DPError) as err:
        dpc.dp_linear_i8(xq, sx, torch.zeros(2, 8, 32, dtype=torch.int8, device="cuda"), torch.zeros(2, 8, device="cuda"))
    assert err.value.code == dpc.DP_ERR_NULL
    with pytest.raises(dpc.DPError) as err:  # K not a multiple of 16
        dpc.dp_linear_i8(xq[:, :24].contiguous(), sx, wq[:, :, :24].contiguous(), sw)
    assert err.value.code == dpc.DP_ERR_SHAPE
    with pytest.raises(dpc.DPError) as err:  # rows off a 16-byte boundary
        dpc.dp_linear_i8(offset_view(xq), sx, wq, sw)
    assert err.value.code == dpc.DP_ERR_SHAPE


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,k,E,K,N,drop,act", [
    (2100, 1, 1, 2064, 2100, 0.0, "tanh"), (6000, 1, 3, 1040, 1500, 0.1, None), (2500, 2, 4, 1600, 1111, 0.0, "tanh"),
    (5000, 1, 2, 3088, 700, 0.5, None)])
def test_many_rows(dtype, T, k, E, K, N, drop, act):
    """Enough rows an expert for the wide tiles: one, two and three chunks of K, ragged tiles both ways, rows past the
    kept ones."""
    dpc = lib()
    assert dpc.dp_linear_i8_work_bytes(T * k, K, N, E) > 0
    r = np.random.default_rng(T + K)
    start = None
    if E > 1:
        start = dpc.dp_route_plan(torch.from_numpy(experts(T, T, k, E, drop)).cuda(), E)[0].cpu().numpy()
    xq, wq = (r.integers(-128, 128, s).astype(np.int8) for s in ((T * k, K), (E, N, K)))
    sx, sw = r.random(T * k).astype(np.float32), r.random((E, N)).astype(np.float32) / (64 * K)
    if start is not None:
        sx[start[-1]:] = np.nan
    check(dpc, xq, sx, wq, sw, r.normal(0, 0.1, (E, N)).astype(np.float32), start, act, dtype)


@pytest.mark.parametrize("K", [8192, 65536])
def test_sums_of_many_rows_are_exact_at_their_largest(K):
    dpc = lib()
    rows, N = 8400, 140 if K == 8192 else 32
    xq, wq = np.full((rows, K), -128, np.int8), np.full((1, N, K), -128, np.int8)
    xq[1::3], wq[0, 1::3] = 127, 127
    xq[2::3, ::2], wq[0, 2::3, 1::2] = 127, 127
    xq[5, 5] = 1
    wq[0, 3] = 0
    wq[0, 3, K - 1] = 1
    assert dpc.dp_linear_i8_work_bytes(rows, K, N, 1) > 0
    one = torch.ones(rows, device="cuda"), torch.ones(1, N, device="cuda")
    y = dpc.dp_linear_i8(torch.from_numpy(xq).cuda(), one[0], torch.from_numpy(wq).cuda(), one[1])
    exact = (xq.astype(np.float64) @ wq[0].astype(np.float64).T).astype(np.float32)  # sums below 2^53
    assert np.array_equal(y.cpu().numpy(), exact)
    again = dpc.dp_linear_i8(torch.from_numpy(xq).cuda(), one[0], torch.from_numpy(wq).cuda(), one[1])
    assert torch.equal(y, again) and dpc.dp_tc_wait_timeouts() == 0
