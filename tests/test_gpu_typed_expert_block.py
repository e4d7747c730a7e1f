"""Embedding, router, experts and norm together, as examples/expert_fitting.py uses them on the compressed model's
descriptors: the whole block's gradient against central differences, and its 4-bit form against the float one."""
import os
import sys

import pytest
import torch

from gpu_common import lib, need_gpu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def ex():
    need_gpu()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import expert_fitting
    return expert_fitting


def typed(ex, score, nexp=6, with_bias=True):
    D = ex.descriptors()
    g = torch.Generator("cuda").manual_seed(5)
    rn = lambda *s: torch.randn(*s, dtype=torch.float64, device="cuda", generator=g)  # noqa: E731
    H = D.shape[1]
    t = ex.TypedBlock(ex.ExpertBlock.random(1, nexp, H, 48), 0.4 * rn(5, H), rn(H, nexp) / H ** 0.5, bias=0.1 * rn(nexp) if with_bias else None, topk=3, score=score)
    types = torch.randint(-1, 5, (D.shape[0],), generator=g, dtype=torch.int32, device="cuda")  # -1: no embedding
    return t, D, types


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
def test_gradient_of_the_block(ex, score, with_bias):
    """E along random directions of the descriptors, the embedding table and the router's weights, the choice unmoved:
    central differences in f64, step 1e-6 (second-order terms and rounding over the step, both below 1e-8 of the
    gradient's magnitudes)."""
    t, D, types = typed(ex, score, with_bias=with_bias)
    E, saved = t.forward(D, types)
    grads = dict(zip(("D", "W", "R"), t.backward(saved)))
    gen = torch.Generator("cuda").manual_seed(4)
    for name, grad in grads.items():
        way = torch.randn(grad.shape, dtype=torch.float64, device="cuda", generator=gen)
        h, e, keep = 1e-6, [], (t.W, t.R)
        for s in (1, -1):
            t.W, t.R = (v + s * h * way if n == name else v for n, v in zip("WR", keep))
            Es, other = t.forward(D + s * h * way if name == "D" else D, types)
            assert torch.equal(other[3], saved[3]), "an expert changed: the direction crosses a border"
            e.append(float(Es))
        t.W, t.R = keep
        assert abs((e[0] - e[1]) / (2 * h) - float((grad * way).sum())) <= 1e-6 * float((grad * way).abs().sum()), name


def test_four_bit_form_is_near(ex):
    """A 4-bit value is off by some 10 % of its size in the mean square (a step of half a unit over 1 to 2, a quarter of a
    unit's step at most, and by up to a quarter above 6), a product of two by 14 %, two layers by 20 %: atomic energies keep
    their order to a correlation of 1 / sqrt(1 + 0.2^2) = 0.98, with room 0.95."""
    t, D, types = typed(ex, "sigmoid")
    u, _, expert, weight = t.choose(D, types)
    b = t.block
    low = ex.ExpertBlock(*(v.float() if isinstance(v, torch.Tensor) else v for v in (b.params, b.widths, b.a, b.w1, b.w2, b.v))).quantise4()
    u, weight = u.float(), weight.float()
    e4 = low.screen4(u, expert, weight)
    _, saved = low.forward(u, expert, weight)
    r2 = saved[8]
    e = (r2 * torch.rsqrt(r2.square().mean(1, keepdim=True) + 1e-6) * low.w2) @ low.v
    assert float(torch.corrcoef(torch.stack([e4, e]))[0, 1]) >= 0.95


def test_block_replays_as_a_graph(ex):
    """Embedding, router, plan, 4-bit layers, combine and norm captured once, replayed on other descriptors and types:
    the eager call's energies, bit for bit."""
    t, D, types = typed(ex, "softmax")
    b = t.block
    f = torch.float32
    t.W, t.R, t.bias = t.W.to(f), t.R.to(f), t.bias.to(f)
    t.block = ex.ExpertBlock(*(v.float() if isinstance(v, torch.Tensor) else v for v in (b.params, b.widths, b.a, b.w1, b.w2, b.v))).quantise4()
    D = D.to(f)

    def energies(D, types):
        u, _, expert, weight = t.choose(D, types)
        return t.block.screen4(u, expert, weight)

    want = energies(D, types)
    Din, tin = torch.zeros_like(D), torch.zeros_like(types)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        energies(Din, tin)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = energies(Din, tin)
    for _ in range(2):
        Din.copy_(D)
        tin.copy_(types)
        graph.replay()
        assert torch.equal(out, want)
        Din.zero_()
        graph.replay()
        assert not torch.equal(out, want)
    assert lib().dp_tc_wait_timeouts() == 0
