"""Experts and weights from a router's logits on the GPU: the choice against one in extended precision, exactly; the
weights and their gradient against 64 bits with elementwise bounds of their arithmetic, and against differences."""
import numpy as np
import pytest
import torch

from gpu_common import lib, need_gpu
from rows_common import IDS, ROWS, SUM_UNIT, TINY, UNIT, f64, offset_view, rnd, within, wtype

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def scores(x, kind):
    """s in long double; a row without a finite largest logit has NaN, masked logits 0."""
    x = x.astype(np.longdouble)
    with np.errstate(all="ignore"):
        if kind == "sigmoid":
            return 1 / (1 + np.exp(-x))
        m = x.max(1, keepdims=True)
        e = np.where(np.isneginf(x), 0, np.exp(x - m))
        return e / e.sum(1, keepdims=True)


def order(v):
    """Columns from the largest on, NaN first, equal ones by index."""
    nan = np.isnan(v)
    return np.lexsort((np.broadcast_to(np.arange(v.shape[1]), v.shape), np.where(nan, 0, -v), ~nan), axis=1)


def reference(x, bias, k, kind, G, keep, top, renorm, scale):
    T, E = x.shape
    s = scores(x, kind)
    c = s if bias is None else s + bias.astype(np.longdouble)
    out = np.isneginf(x) if bias is None else np.isneginf(x) | np.isneginf(bias)
    c = np.where(out, -np.inf, c)
    by = np.where(out, -np.inf, x.astype(np.longdouble)) if bias is None else c
    if keep < G:
        per = E // G
        of = (by if bias is None and (top == 1 or per == 1) else c).reshape(T, G, per)
        best = -np.sort(-of, 2) if not np.isnan(of).any() else np.take_along_axis(of, order(of.reshape(T * G, per)).reshape(of.shape), 2)
        g = best[:, :, 0].copy()
        if top == 2 and per > 1:
            two = ~np.isneginf(best[:, :, 1])
            g[two] += best[:, :, 1][two]
        kept = np.zeros((T, G), bool)
        np.put_along_axis(kept, order(g)[:, :keep], True, 1)
        by = np.where(np.repeat(kept, per, 1), by, -np.inf)
    e = order(by)[:, :k]
    have = ~np.isneginf(np.take_along_axis(by, e, 1))
    w = np.take_along_axis(s, e, 1)
    if renorm:
        xe = np.where(have, np.take_along_axis(x, e, 1).astype(np.longdouble), -np.inf)
        with np.errstate(all="ignore"):
            # log s up to a constant of the row: nothing underflows
            ls = xe if kind == "softmax" else np.where(xe < 0, xe - np.log1p(np.exp(xe)), -np.log1p(np.exp(-xe)))
            w = np.where(have, np.exp(ls - np.where(have, ls, -np.inf).max(1, keepdims=True)), 0)
            w = w / w.sum(1, keepdims=True)
    return np.where(have, e, -1), np.where(have, scale * w, 0).astype(np.float64)


def weight_bound(x, E, k, renorm, dtype):
    """Relative: twice an exponential's 2 ulp (4 units) and its argument's rounding (the spread of the logits in units),
    the sum's E or k roundings, and a few of quotients and products."""
    fin = np.where(np.isfinite(x), x, 0)
    spread = np.minimum(fin.max(1) - fin.min(1), 110)[:, None] if dtype != torch.float64 else np.minimum(fin.max(1) - fin.min(1), 750)[:, None]
    return (20 + 2 * spread + (k if renorm else E)) * SUM_UNIT[dtype]


# E over every split of lanes and its ends; k to the most
CASES = [(1, 1, 1, 1, 1, 1), (5, 2, 2, 1, 1, 1), (33, 8, 2, 1, 1, 1), (200, 8, 4, 4, 2, 2), (50, 8, 8, 4, 4, 2), (64, 13, 3, 1, 1, 1), (70, 32, 5, 4, 3, 1),
         (70, 33, 5, 3, 2, 2), (500, 61, 3, 1, 1, 1), (300, 128, 6, 8, 4, 2), (300, 128, 64, 2, 1, 1), (100, 129, 8, 43, 20, 2),
         (60, 500, 8, 4, 1, 2), (40, 512, 64, 1, 1, 1), (40, 513, 20, 27, 3, 1), (30, 1024, 8, 1024, 9, 2), (30, 1024, 64, 16, 2, 2), (0, 8, 2, 1, 1, 1)]


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,E,k,G,keep,top", CASES)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("variant", ["plain", "bias", "renorm", "bias-renorm"])
def test_choice_and_weights(dtype, T, E, k, G, keep, top, kind, variant):
    dpc = lib()
    x, xr = rnd(T + E, T, E, dtype=dtype, scale=1.5)
    b, br = rnd(E + 3, E, dtype=wtype(dtype), scale=0.05) if "bias" in variant else (None, None)
    renorm = "renorm" in variant
    args = dict(bias=b, score=kind, ngroup=G, keep_groups=keep, group_top=top, renorm=renorm, scale=1.75)
    e, w = dpc.dp_route_topk(x, k, **args)
    re, rw = reference(xr, br, k, kind, G, keep, top, renorm, 1.75)
    assert e.dtype == torch.int32 and w.dtype == wtype(dtype)
    assert np.array_equal(e.cpu().numpy(), re)
    within(w, rw, np.abs(rw) * weight_bound(xr, E, k, renorm, dtype) if T else 0.0, "w")
    e2, w2 = dpc.dp_route_topk(offset_view(x), k, **{**args, "bias": None if b is None else offset_view(b)})
    assert torch.equal(e, e2) and torch.equal(w, w2)


@pytest.mark.parametrize("dtype", ROWS[1:], ids=IDS[1:])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("G,keep,top", [(1, 1, 1), (4, 2, 2), (4, 2, 1), (12, 5, 2), (24, 7, 2)])
@pytest.mark.parametrize("k", [2, 6, 8, 9, 12])
def test_scores_nearer_than_f32_tells_apart(dtype, kind, G, keep, top, k):
    """A bias of C - s, rounded to f32, makes all scores of a row differ by roundings alone: the choice is still that of
    exact arithmetic.  The reference's own neighbours differ by more than its error (64 bits of mantissa)."""
    dpc = lib()
    T, E = 40, 48
    x, xr = rnd(5, 1, E, dtype=dtype)
    x, xr = x.expand(T, E).contiguous(), np.broadcast_to(xr, (T, E))
    s = scores(xr, kind)[0]
    b = torch.from_numpy((1.0 - s).astype(np.float64)).to(wtype(dtype)).cuda()
    br = f64(b)
    c = np.sort(s + br)
    assert np.diff(c).max() < 2.0 ** -20
    assert np.diff(c).min() > 2.0 ** -50
    e, _ = dpc.dp_route_topk(x, k, bias=b, score=kind, ngroup=G, keep_groups=keep, group_top=top)
    re, _ = reference(xr, br, k, kind, G, keep, top, True, 1.0)
    assert np.array_equal(e.cpu().numpy(), re)


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("E,G,keep", [(8, 1, 1), (60, 1, 1), (60, 6, 2), (200, 4, 2)])
def test_equal_scores_go_by_index(dtype, kind, with_bias, E, G, keep):
    dpc = lib()
    b = torch.zeros(E, dtype=wtype(dtype), device="cuda") if with_bias else None
    for value in (0.0, -3.0, float(torch.finfo(dtype).min), float(torch.finfo(dtype).max), 40.0):
        x = torch.full((3, E), value, dtype=dtype, device="cuda")
        x[1, E // 2] = -0.0 if value == 0.0 else value
        e, w = dpc.dp_route_topk(x, 4, bias=b, score=kind, ngroup=G, keep_groups=keep)
        assert e.tolist() == [[0, 1, 2, 3]] * 3, value
        assert torch.equal(w, torch.full_like(w, 0.25))
    # coarse logits: most rows hold ties
    g = np.random.default_rng(3).integers(-2, 3, (400, E)).astype(np.float64)
    e, _ = dpc.dp_route_topk(torch.from_numpy(g).to(dtype).cuda(), 4, bias=b, score=kind, ngroup=G, keep_groups=keep)
    # equal logits give equal scores, so the reference's order is that of the logits
    re, _ = reference(g, None if b is None else np.zeros(E), 4, kind, G, keep, 2, True, 1.0)
    assert np.array_equal(e.cpu().numpy(), re)


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("E,G,keep", [(9, 1, 1), (36, 6, 3), (1000, 10, 4)])
def test_masks_infinities_and_nan(dtype, kind, renorm, E, G, keep):
    dpc = lib()
    inf, nan, low = float("inf"), float("nan"), float(torch.finfo(dtype).min)
    x, _ = rnd(E, 12, E, dtype=dtype)
    x[0] = -inf                      # nothing left
    x[1, 1:] = -inf                  # one left
    x[2, : E - 2] = -inf             # two
    x[3, ::2] = low                  # the type's lowest value is a number
    x[4] = low
    x[5, 3] = nan
    x[6] = nan
    x[7, 2] = inf
    x[8, :4] = inf
    x[9, 5], x[9, 1] = nan, -inf
    b = torch.zeros(E, dtype=wtype(dtype), device="cuda")
    b[0] = -inf
    for bias in (None, b):
        e, w = dpc.dp_route_topk(x, 3, bias=bias, score=kind, ngroup=G, keep_groups=keep, renorm=renorm, scale=2.0)
        re, rw = reference(f64(x), None if bias is None else f64(bias), 3, kind, G, keep, 2, renorm, 2.0)
        rows = [0, 1, 2, 3, 10, 11]
        if G == 1 or kind == "sigmoid":  # a softmax row with a NaN or +inf has NaN in all scores
            rows += [4]
        assert np.array_equal(e.cpu().numpy()[rows], re[rows])
        within(w[rows], rw[rows], np.abs(rw[rows]) * weight_bound(f64(x)[rows], E, 3, renorm, dtype) + 2.0 ** -126, "w")
        e, w = e.cpu().numpy(), f64(w)
        assert (e[0] == -1).all() and (w[0] == 0).all()
        if bias is None:
            assert list(e[1]) == [0, -1, -1] and w[1, 1] == w[1, 2] == 0
            assert sorted(e[2][:2]) == [E - 2, E - 1] and e[2, 2] == -1
            assert e[5, 0] == 3 if kind == "sigmoid" or G == 1 else True
            assert list(e[6]) == [0, 1, 2]
        else:
            assert (e[1] == -1).all() and (e != 0).all()
        assert np.isnan(w[6]).all() and np.isnan(w[5]).any() and (e[9] != 1).all() and np.isnan(w[9]).any()
        if kind == "softmax":
            assert np.isnan(w[7]).any() and np.isnan(w[8]).any()


def gradient(x, e, dw, kind, renorm, scale):
    """(dx, magnitudes) in f64 from the formulas, pair by pair."""
    T, E = x.shape
    s = scores(x, kind).astype(np.float64)
    dx, mag = np.zeros((T, E)), np.zeros((T, E))
    for t in range(T):
        js = [j for j in range(e.shape[1]) if 0 <= e[t, j] < E and not np.isneginf(x[t, e[t, j]])]
        ids = [e[t, j] for j in js]
        if not js:
            continue
        xe = x[t, ids]
        if renorm:
            ls = xe if kind == "softmax" else np.where(xe < 0, xe - np.log1p(np.exp(-np.abs(xe))), -np.log1p(np.exp(-np.abs(xe))))
            n = np.exp(ls - ls.max())
            n /= n.sum()
            d = scale * dw[t, js]
            co, cm = n * (d - (n * d).sum()), n * (np.abs(d) + (n * np.abs(d)).sum())
        else:
            co = scale * dw[t, js] * s[t, ids]
            cm = np.abs(co)
        if kind == "sigmoid":
            one_less = 1 / (1 + np.exp(np.minimum(xe, 700)))
            co, cm = co * one_less, cm * one_less
        np.add.at(dx[t], ids, co)
        np.add.at(mag[t], ids, cm)
        if kind == "softmax" and not renorm:
            dx[t] -= s[t] * co.sum()
            mag[t] += s[t] * cm.sum()
    return dx, mag


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (5, 2, 2), (33, 8, 2), (40, 32, 32), (33, 61, 3), (20, 128, 6), (20, 128, 64), (9, 300, 64), (9, 513, 7), (9, 1024, 8), (0, 4, 2)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient(dtype, T, E, k, kind, renorm):
    """Bounds as the weights', on the magnitudes of what is added; ids of no expert, masked logits and one expert twice
    among the pairs; every element is written."""
    dpc = lib()
    r = np.random.default_rng(E + k)
    x, xr = rnd(T + E + 1, T, E, dtype=dtype, scale=1.5)
    e = np.stack([r.permutation(E)[:k] for _ in range(T)]) if T else np.zeros((0, k), np.int64)
    if T > 4 and k > 1:
        e[0, 1] = e[0, 0]
        e[1, 0], e[2, 1], e[3, 0] = -1, E, -2 ** 31
        x[4, e[4, 0]] = -float("inf")
        xr[4, e[4, 0]] = -np.inf
    if T > 8:
        e[5], x[6], xr[6] = -1, -float("inf"), -np.inf
    dw, dwr = rnd(9, T, k, dtype=wtype(dtype))
    et = torch.from_numpy(e.astype(np.int32)).cuda()
    out = torch.full_like(x, float("nan"))
    dx = dpc.dp_route_topk_grad(x, et, dw, score=kind, renorm=renorm, scale=1.75, out=out)
    assert dx is out
    ref, mag = gradient(xr, e, dwr, kind, renorm, 1.75)
    b = mag * ((60 + E + 4 * k) * SUM_UNIT[dtype] + 4 * np.minimum(np.ptp(np.where(np.isfinite(xr), xr, 0), 1), 110)[:, None] * SUM_UNIT[dtype] if T else 0)
    within(dx, ref, b + np.abs(ref) * UNIT[dtype] * 1.01 + TINY[dtype], "dx")
    dx2 = dpc.dp_route_topk_grad(offset_view(x), et, dw, score=kind, renorm=renorm, scale=1.75)
    assert torch.equal(dx, dx2)


@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_gradient_is_the_weights_differences(kind, renorm):
    """Central differences of sum(w v) in f64, the choice unmoved: error h^2 max|third derivative| / 6 (below 6 scale |v|
    for these scores) and rounding 2^-52 / h."""
    dpc = lib()
    T, E, k, h = 6, 21, 4, 1e-4
    x, _ = rnd(3, T, E, scale=1.0)
    x += 0.01 * torch.arange(E, dtype=torch.float64, device="cuda")
    v, _ = rnd(4, T, k)
    kw = dict(score=kind, renorm=renorm, scale=1.5)
    e, _ = dpc.dp_route_topk(x, k, **kw)
    dx = dpc.dp_route_topk_grad(x, e, v, **kw)
    num = torch.zeros_like(dx)
    for i in range(E):
        step = torch.zeros_like(x)
        step[:, i] = h
        (e1, w1), (e0, w0) = dpc.dp_route_topk(x + step, k, **kw), dpc.dp_route_topk(x - step, k, **kw)
        assert torch.equal(e1, e) and torch.equal(e0, e)
        num[:, i] = ((w1 - w0) * v).sum(1) / (2 * h)
    bound = 1.5 * f64(v.abs().sum(1))[:, None] * (6 * h * h / 6 + 200 * 2.0 ** -52 / h)
    within(dx, f64(num), np.broadcast_to(bound, (T, E)), "dx")


def test_many_tokens_streams_and_graph():
    """More tokens than blocks run at once; on a side stream; captured and replayed on new logits, the outputs in place."""
    dpc = lib()
    T, E, k = 70001, 64, 4
    x, xr = rnd(8, T, E, dtype=torch.bfloat16)
    b, br = rnd(9, E, dtype=torch.float32, scale=0.1)
    kw = dict(bias=b, score="sigmoid", ngroup=8, keep_groups=3, scale=2.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        e, w = dpc.dp_route_topk(x, k, **kw)
    torch.cuda.current_stream().wait_stream(side)
    re, rw = reference(xr[:2000], br, k, "sigmoid", 8, 3, 2, True, 2.5)
    assert np.array_equal(e[:2000].cpu().numpy(), re)
    tail, _ = reference(xr[-500:], br, k, "sigmoid", 8, 3, 2, True, 2.5)
    assert np.array_equal(e[-500:].cpu().numpy(), tail)
    dw, _ = rnd(10, T, k, dtype=torch.float32)
    dx = dpc.dp_route_topk_grad(x, e, dw, score="sigmoid", scale=2.5)
    out = torch.empty_like(e), torch.empty_like(w)
    gout = torch.empty_like(dx)
    xs = torch.zeros_like(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dpc.dp_route_topk(xs, k, out=out, **kw)
        dpc.dp_route_topk_grad(xs, out[0], dw, score="sigmoid", scale=2.5, out=gout)
    xs.copy_(x)
    graph.replay()
    assert torch.equal(out[0], e) and torch.equal(out[1], w) and torch.equal(gout, dx)


@pytest.mark.parametrize("E,k", [(60, 3), (200, 8), (1000, 8), (1000, 20), (1024, 64)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("sign", [1, -1])
def test_f32_logits_that_share_their_upper_bits(E, k, kind, sign):
    """Neighbouring floats in any order: what a key shortened by the expert's index cannot tell apart, without a bias and
    with one that is the same for all (scores equal in f32, logits not)."""
    dpc = lib()
    r = np.random.default_rng(E + k)
    v = np.stack([r.permutation(E) for _ in range(50)]).astype(np.float64)
    x = torch.from_numpy(sign * (1.0 + v * 2.0 ** -23)).float().cuda()
    want = np.argsort(-sign * v, axis=1)[:, :k]
    e, _ = dpc.dp_route_topk(x, k, score=kind)
    assert np.array_equal(e.cpu().numpy(), want)
    b = torch.full((E,), 0.25, device="cuda")
    e, _ = dpc.dp_route_topk(x, k, bias=b, score=kind)
    assert np.array_equal(e.cpu().numpy(), want)


@pytest.mark.parametrize("T", [1, 3, 4, 5, 15, 16, 17, 33])
def test_few_close_pairs_among_clear_ones(T):
    """Two of a token's best scores closer than f32 holds, the others apart: at each place of the order, at its end, and in
    tokens beside others that need nothing."""
    dpc = lib()
    E, k = 40, 5
    r = np.random.default_rng(T)
    for place in range(k + 1):
        c = np.sort(r.uniform(0.2, 0.9, (T, E)), axis=1)[:, ::-1].copy()
        c[:, :10] += np.linspace(1.0, 0.1, 10)  # clear gaps among the best
        # a logit's f32 neighbours differ by more than f32 scores near 1 do
        lo = torch.full((T, E), -3.0)
        x = lo + 0.1 * torch.from_numpy(r.normal(size=(T, E))).float()
        b = torch.zeros(E)
        order_ = r.permutation(E)
        b[order_] = torch.from_numpy(c[0]).float()
        x = x[:1].expand(T, E).contiguous()
        s0 = scores(x.double().numpy(), "sigmoid")[0]
        # the pair: equal c but for the bias's rounding
        i, j = order_[place], order_[place + 1]
        b[j] = float(np.float32(float(s0[i]) + float(b[i]) - float(s0[j])))
        e, w = dpc.dp_route_topk(x.cuda(), k, bias=b.cuda(), score="sigmoid")
        re, rw = reference(x.double().numpy(), b.double().numpy(), k, "sigmoid", 1, 1, 1, True, 1.0)
        assert np.array_equal(e.cpu().numpy(), re), place
        within(w, rw, np.abs(rw) * weight_bound(x.double().numpy(), E, k, True, torch.float32), "w")
