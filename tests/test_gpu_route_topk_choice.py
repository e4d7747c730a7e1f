"""Rows on which the router's choice hangs on scores with errors of very different size, on sums that cancel, or on
ties at the border: against extended precision, exactly."""
import numpy as np
import pytest
import torch

from gpu_common import lib, need_gpu
from test_gpu_route_topk import reference, scores

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def logit(p):
    p = p.astype(np.longdouble)
    return np.log(p) - np.log1p(-p)


def cancelling(seed, T, E, k, close):
    """(x, b) f32, sigmoid: k - 1 clear best ones, then A and B without a bias, clearly apart, and C, whose score near 1
    its bias cancels to slightly more than A's: in f32 C is a multiple of 2^-24, often below both.  close: two of the best
    ones share their upper bits, so that the shortened keys alone do not settle the token."""
    r = np.random.default_rng(seed)
    b = np.zeros(E, np.float32)
    at = r.permutation(E)
    best, (A, B, C) = at[:k - 1], at[k - 1: k + 2]
    b[C] = np.float32(-0.9634783)
    x = np.full((T, E), -14.0, np.float32) - r.random((T, E)).astype(np.float32)
    x[:, best] = (-4.0 + 0.5 * np.arange(k - 1) + 0.1 * r.random((T, k - 1))).astype(np.float32)
    if close and k > 2:
        x[:, best[1]] = x[:, best[0]] * np.float32(1 - 2.0 ** -19)
    x[:, A] = (-10.0 - 0.02 * r.random(T)).astype(np.float32)
    x[:, B] = x[:, A] - np.float32(1e-4)
    s = lambda v: 1 / (1 + np.exp(-v.astype(np.longdouble)))  # noqa: E731
    cA = s(x[:, A])
    # the f32 logit of C whose score lies closest above the wanted one
    want = cA + (0.2 + 0.8 * r.random(T)) * 2.0 ** -26 - np.longdouble(b[C])
    x[:, C] = logit(want).astype(np.float32)
    x[:, C] = np.where(s(x[:, C]) + np.longdouble(b[C]) <= cA, np.nextafter(x[:, C], np.float32(9)), x[:, C])
    return x, b


@pytest.mark.parametrize("E,k", [(4, 1), (8, 3), (40, 5), (128, 6), (130, 8), (60, 9), (128, 20), (300, 12), (100, 40), (300, 64), (1000, 8), (1000, 30)])
@pytest.mark.parametrize("close", [False, True])
def test_an_error_larger_than_the_borders_own(E, k, close):
    dpc = lib()
    T = 400
    x, b = cancelling(E + k, T, E, k, close)
    e, _ = dpc.dp_route_topk(torch.from_numpy(x).cuda(), k, bias=torch.from_numpy(b).cuda(), score="sigmoid")
    re, _ = reference(x.astype(np.float64), b.astype(np.float64), k, "sigmoid", 1, 1, 1, True, 1.0)
    assert np.array_equal(e.cpu().numpy(), re)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k,G,keep", [(24, 2, 1, 1), (24, 6, 4, 2), (96, 8, 1, 1), (96, 8, 6, 3), (96, 10, 1, 1), (96, 10, 4, 3), (600, 8, 1, 1), (600, 40, 4, 3)])
def test_biases_that_cancel_scores(dtype, kind, E, k, G, keep):
    """Half of the experts with a bias near the negative of their score, so that all c are small and the errors of two
    neighbours are unlike."""
    dpc = lib()
    r = np.random.default_rng(E + k)
    T = 200
    x = torch.from_numpy(r.normal(size=(1, E)) * 2.0).to(dtype)
    x = (x.expand(T, E) + torch.from_numpy(r.integers(0, 2, (T, E)) * 2.0 ** -9)).to(dtype)
    s = scores(x.double().numpy(), kind)
    b = np.where(r.random(E) < 0.5, -s[0] + 2.0 ** -14 * r.random(E), 0.0).astype(np.float32)
    small = np.argsort(-s[0])
    b[small[: E // 4]] = (-s[0] + 2.0 ** -14 * r.random(E))[small[: E // 4]].astype(np.float32)
    e, _ = dpc.dp_route_topk(x.cuda(), k, bias=torch.from_numpy(b).cuda(), score=kind, ngroup=G, keep_groups=keep)
    re, _ = reference(x.double().numpy(), b.astype(np.float64), k, kind, G, keep, 2, True, 1.0)
    assert np.array_equal(e.cpu().numpy(), re)


@pytest.mark.parametrize("E,k", [(5, 1), (40, 1), (40, 5), (128, 7), (128, 8), (60, 9), (300, 20), (200, 33)])
@pytest.mark.parametrize("same", [2, 3, 9, 12])
@pytest.mark.parametrize("bias", [None, 0.0, 0.25])
def test_equal_ones_at_the_border_before_a_larger_one(E, k, same, bias):
    """Equal scores on both sides of the border and, by a shortened key, equal to a larger one of a higher index."""
    if k - 1 + same >= E:
        pytest.skip("more equal ones than experts")
    dpc = lib()
    x = np.full((3, E), -2.0, np.float32)
    x[:, : k - 1] = 3.0 + 0.25 * np.arange(k - 1)
    x[:, k - 1: k - 1 + same] = 1.0
    x[0, k - 1 + same] = np.float32(1 + 2.0 ** -23)
    x[1, k - 1 + same] = np.float32(1 + 2.0 ** -21)
    b = None if bias is None else torch.full((E,), bias, device="cuda")
    e, _ = dpc.dp_route_topk(torch.from_numpy(x).cuda(), k, bias=b, score="sigmoid")
    # one bias for all: the order of the logits
    re, _ = reference(x.astype(np.float64), None, k, "sigmoid", 1, 1, 1, True, 1.0)
    assert np.array_equal(e.cpu().numpy(), re)


@pytest.mark.parametrize("E,k", [(2, 1), (40, 1), (40, 3), (40, 12), (300, 40)])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
def test_scores_below_the_normal_range(E, k, kind):
    """Scores of 2^-126.5 and biases of 2^-127: no relative bound holds for what the hardware's exponential flushes."""
    dpc = lib()
    x = np.full((2, E), -104.0, np.float32)
    b = np.zeros(E, np.float32)
    x[:, 0], x[:, 1], b[0] = -97.0, -87.68, 2.0 ** -127
    x[1, :2], b[1] = x[1, 1::-1], 0.0
    if E > 2:  # what the others lie under
        x[:, 2] = 0.0
        b[2] = -np.inf
    elif kind == "softmax":
        pytest.skip("a softmax of these alone is near 1")
    e, _ = dpc.dp_route_topk(torch.from_numpy(x).cuda(), k, bias=torch.from_numpy(b).cuda(), score=kind)
    re, _ = reference(x.astype(np.float64), b.astype(np.float64), k, kind, 1, 1, 1, True, 1.0)
    assert np.array_equal(e.cpu().numpy(), re)


@pytest.mark.parametrize("dtype", [torch.float64, torch.float32, torch.bfloat16, torch.float16], ids=["f64", "f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k,G,keep", [(2, 1, 1, 1), (30, 4, 1, 1), (30, 8, 1, 1), (30, 8, 5, 2), (128, 6, 8, 4), (128, 12, 1, 1), (128, 12, 8, 4), (1000, 50, 1, 1), (1000, 8, 10, 2)])
@pytest.mark.parametrize("value", [0.0, 0.5, -3.0])
def test_one_bias_for_all_keeps_the_order_of_the_logits(dtype, kind, E, k, G, keep, value):
    """Sigmoids of 40 and 45 are both 1 in f64, a softmax's 1e-20 vanishes beside 0.5: a bias that is the same for all
    changes no choice, nor do groups scored by their best one."""
    dpc = lib()
    r = np.random.default_rng(E + k)
    x = torch.from_numpy(np.concatenate([r.uniform(-60, 60, (20, E)), r.uniform(35, 60, (20, E)), np.round(r.uniform(38, 44, (20, E)))])).to(dtype)
    x[0, :2] = torch.tensor([40.0, 45.0]).to(dtype)
    b = torch.full((E,), value, dtype=torch.float64 if dtype == torch.float64 else torch.float32, device="cuda")
    kw = dict(score=kind, ngroup=G, keep_groups=keep, group_top=1)
    e, w = dpc.dp_route_topk(x.cuda(), k, bias=b, **kw)
    if G > 1:  # groups whose best scores are equal in f64 go by the lowest index: those that differ there
        x64 = x.double()
        s = torch.sigmoid(x64) if kind == "sigmoid" else torch.softmax(x64, 1)
        best = (s.view(-1, G, E // G).amax(2) + b.double().cpu()[0]).sort(1).values
        clear = (best.diff(dim=1) > 1e-10 * best[:, 1:].abs()).all(1).numpy()
    else:
        clear = np.ones(x.shape[0], bool)
    re, _ = reference(x.double().numpy(), None, k, kind, G, keep, 1, True, 1.0)
    assert np.array_equal(e.cpu().numpy()[clear], re[clear])
