"""Embedding of ids and its gradient on the GPU: the plan against a stable sort, rows and gradients against 64 bits with
elementwise bounds of their arithmetic."""
import numpy as np
import pytest
import torch

from gpu_common import lib, need_gpu
from rows_common import IDS, ROWS, SUM_UNIT, TINY, UNIT, f64, offset_view, rnd, within, wtype

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def ids_of(seed, T, V, drop=0.1, skew=True):
    r = np.random.default_rng(seed)
    v = np.minimum((V ** r.random(T)).astype(np.int64), V) - 1 if skew else r.integers(0, V, T)
    v = r.permutation(V)[v]
    bad = r.choice(np.array([-1, -2 ** 31, V, V + 7, 2 ** 31 - 1]), T)
    return np.where(r.random(T) < drop, bad, v).astype(np.int32)


def plan(ids, V):
    key = np.where((ids >= 0) & (ids < V), ids.astype(np.int64), V)
    at = np.argsort(key, kind="stable")
    return np.searchsorted(key[at], np.arange(V + 1)), np.where(key[at] < V, at, -1)


@pytest.mark.parametrize("T,V,drop", [
    (0, 1, 0.0), (1, 1, 0.0), (1, 70000, 0.0), (33, 4, 0.3), (4095, 255, 0.1), (4096, 256, 0.0), (4096, 100000, 0.1), (4097, 4, 0.0), (4097, 255, 0.2),
    (9001, 2, 1.0), (32768, 65535, 0.1), (32769, 65536, 0.1), (65537, 118, 0.0), (131073, 1000, 0.05), (70001, 1 << 20, 0.05), (300007, (1 << 24) - 1, 0.1), (1500001, 30011, 0.1)])
def test_plan(T, V, drop):
    dpc = lib()
    i = ids_of(T + V, T, V, drop)
    t = torch.from_numpy(i).cuda()
    start, src = dpc.dp_embed_plan(t, V)
    rs, rr = plan(i, V)
    assert start.dtype == torch.int64 and src.dtype == torch.int32
    assert np.array_equal(start.cpu().numpy(), rs)
    assert np.array_equal(src.cpu().numpy(), rr)
    if V <= 1024:
        s2, r2, _ = dpc.dp_route_plan(t[:, None], V)
        assert torch.equal(start, s2) and torch.equal(src, r2)


@pytest.mark.parametrize("T,V", [(5000, 7), (5000, 70000)])
def test_plan_of_equal_and_reversed_ids(T, V):
    dpc = lib()
    start, src = dpc.dp_embed_plan(torch.full((T,), V - 1, dtype=torch.int32, device="cuda"), V)
    assert int(start[V - 1]) == 0 and int(start[V]) == T and torch.equal(src, torch.arange(T, dtype=torch.int32, device="cuda"))
    i = (np.arange(T)[::-1] * (V // 7 if V < T else 1) % V).astype(np.int32)
    start, src = dpc.dp_embed_plan(torch.from_numpy(i).cuda(), V)
    rs, rr = plan(i, V)
    assert np.array_equal(start.cpu().numpy(), rs) and np.array_equal(src.cpu().numpy(), rr)


SHAPES = [(1, 1, 1), (4, 118, 240), (37, 3, 17), (200, 5, 1600), (64, 90, 1003), (5, 4, 5000), (300, 2, 4), (0, 3, 16), (3000, 700, 64), (20, 1, 2056)]


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,V,H", SHAPES)
@pytest.mark.parametrize("offset", [0, 1])
def test_rows(dtype, T, V, H, offset):
    """One fused product and sum in the accumulation type, then one rounding to the row type."""
    dpc = lib()
    i = ids_of(T + H, T, V, 0.2)
    (W, Wr), (add, ar) = rnd(1, V, H, dtype=dtype), rnd(2, T, H, dtype=dtype)
    ids = torch.from_numpy(i).cuda()
    if offset:
        W, add, ids = offset_view(W), offset_view(add), offset_view(ids)
    have = (i >= 0) & (i < V)
    emb = np.where(have[:, None], 1.75 * Wr[np.where(have, i, 0)], 0.0)
    for a, ref in ((None, emb), (add, ar + emb)):
        y = dpc.dp_embed_fwd(W, ids, scale=1.75, add=a)
        # (the reference rounds its product too)
        within(y, ref, np.abs(ref) * (UNIT[dtype] + SUM_UNIT[dtype]) * 1.001 + np.abs(emb) * 2.0 ** -53 + TINY[dtype], "y")
    y0 = dpc.dp_embed_fwd(W, ids, scale=1.75, add=add)
    assert torch.equal(dpc.dp_embed_fwd(W, ids, scale=1.75, add=add, out=add), y0)  # in place
    # unscaled rows are copies, NaN and infinities with them; rows without an id are add's bits
    if T:
        W[0, 0], add[0, 0] = float("nan"), float("inf")
        y = dpc.dp_embed_fwd(W, ids)
        assert torch.equal(torch.nan_to_num(y[torch.from_numpy(have).cuda()]), torch.nan_to_num(W[ids.long()[torch.from_numpy(have).cuda()]]))
        y = dpc.dp_embed_fwd(W, ids, add=add)
        none = torch.from_numpy(~have).cuda()
        assert torch.equal(y[none], add[none])


GRADS = SHAPES + [(2000, 1, 33), (5000, 4, 240), (9973, 3, 1003), (4099, 3000, 130), (70000, 2, 8), (1025, 2, 9000), (40000, 118, 64)]


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,V,H", GRADS)
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(dtype, T, V, H, accumulate):
    """Sums of n_v rows: at most n_v + 2 roundings of the sums' type on the sum of magnitudes, in any order."""
    dpc = lib()
    i = ids_of(T + H, T, V, 0.15, skew=V > 4)
    dy, dyr = rnd(3, T, H, dtype=dtype)
    W0, W0r = rnd(4, V, H, dtype=wtype(dtype))
    ids = torch.from_numpy(i).cuda()
    start, src = dpc.dp_embed_plan(ids, V)
    out = W0.clone() if accumulate else torch.full_like(W0, float("nan"))
    if T:  # tokens without an id are not read
        dy[torch.from_numpy((i < 0) | (i >= V)).cuda()] = float("nan")
    have = np.flatnonzero((i >= 0) & (i < V))
    ref, mag = (W0r.copy(), np.abs(W0r)) if accumulate else (np.zeros((V, H)), np.zeros((V, H)))
    at = have[np.argsort(i[have], kind="stable")]
    if at.size:
        first = np.flatnonzero(np.r_[True, np.diff(i[at]) != 0])
        ref[i[at][first]] += 1.75 * np.add.reduceat(dyr[at], first, 0)
        mag[i[at][first]] += 1.75 * np.add.reduceat(np.abs(dyr[at]), first, 0)
    n = np.bincount(i[have], minlength=V)[:, None]
    dW = dpc.dp_embed_grad(dy, ids, start, src, scale=1.75, out=out, accumulate=accumulate)
    assert dW is out and dW.dtype == wtype(dtype)
    # the reference's own sums have as many roundings of 2^-53
    within(dW, ref, mag * (n + 3) * (SUM_UNIT[dtype] + 2.0 ** -53), "dW")
    if accumulate:
        assert torch.equal(dW[torch.from_numpy(n[:, 0] == 0).cuda()], W0[torch.from_numpy(n[:, 0] == 0).cuda()])
    else:
        assert not dW[torch.from_numpy(n[:, 0] == 0).cuda()].any()
    again = dpc.dp_embed_grad(offset_view(dy), ids, start, src, scale=1.75, out=W0.clone(), accumulate=accumulate)
    within(again, ref, mag * (n + 3) * (SUM_UNIT[dtype] + 2.0 ** -53), "dW of a view")
    twice = dpc.dp_embed_grad(dy, ids, start, src, scale=1.75, out=W0.clone(), accumulate=accumulate)
    assert torch.equal(dW, twice)


def test_gradient_is_the_rows_differences():
    """sum(y v) is linear in W: differences of f64 rows are exact but for roundings."""
    dpc = lib()
    T, V, H = 50, 6, 12
    i = ids_of(1, T, V, 0.1)
    ids = torch.from_numpy(i).cuda()
    W, _ = rnd(1, V, H)
    v, vr = rnd(2, T, H)
    start, src = dpc.dp_embed_plan(ids, V)
    dW = f64(dpc.dp_embed_grad(v, ids, start, src, scale=0.7))
    base = (dpc.dp_embed_fwd(W, ids, scale=0.7) * v).sum()
    for r, c in ((0, 0), (3, 7), (5, 11)):
        W2 = W.clone()
        W2[r, c] += 1.0
        diff = float((dpc.dp_embed_fwd(W2, ids, scale=0.7) * v).sum() - base)
        assert abs(diff - dW[r, c]) <= 2.0 ** -53 * 4 * T * H * 10 * np.abs(vr).max()


@pytest.mark.parametrize("T,V,H", [(30000, 4, 240), (3000, 5000, 100)])
def test_graph_and_streams(T, V, H):
    """Plan and gradient captured with buffers of their own and replayed on other ids, and two of them at once."""
    dpc = lib()
    a, b = (torch.from_numpy(ids_of(s, T, V)).cuda() for s in (1, 2))
    dy, _ = rnd(3, T, H, dtype=torch.float32)
    want = {}
    for n, i in (("a", a), ("b", b)):
        start, src = dpc.dp_embed_plan(i, V)
        want[n] = start, src, dpc.dp_embed_grad(dy, i, start, src)
    ids = torch.zeros_like(a)
    out = [torch.empty_like(t) for t in want["a"]]
    pw = torch.empty(dpc.dp_embed_plan_work_bytes(T, V), dtype=torch.uint8, device="cuda")
    gw = torch.empty(dpc.dp_embed_grad_work_bytes(T, H, torch.float32), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dpc.dp_embed_plan(ids, V, out=out[:2], work=pw)
        dpc.dp_embed_grad(dy, ids, out[0], out[1], out=out[2], work=gw)
    for n, i in (("a", a), ("b", b), ("a", a)):
        ids.copy_(i)
        graph.replay()
        for got, ref in zip(out, want[n]):
            assert torch.equal(got, ref)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for st, i in zip(streams, (a, b)):
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            for _ in range(5):
                start, src = dpc.dp_embed_plan(i, V)
                dW = dpc.dp_embed_grad(dy, i, start, src)
            got.append((start, src, dW))
    torch.cuda.synchronize()
    for g, n in zip(got, "ab"):
        for x, y in zip(g, want[n]):
            assert torch.equal(x, y)
