"""The expert-block calls together, as examples/expert_fitting.py uses them on the compressed model's descriptors:
the whole block's gradient against central differences, and its 8-bit form against the float one."""
import os
import sys

import pytest
import torch

from gpu_common import need_gpu

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def ex():
    need_gpu()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import expert_fitting
    return expert_fitting


def setup(ex, nexp=5, drop=False):
    u = ex.descriptors()
    g = torch.Generator("cuda").manual_seed(3)
    expert, weight = ex.route(torch.randn(u.shape[0], nexp, dtype=torch.float64, device="cuda", generator=g), 2)
    if drop:
        expert[::7, 1] = -1
        expert[3] = -1  # an atom without any net: only its residual stream
    gate = torch.rand(u.shape[0], dtype=torch.float64, device="cuda", generator=g)
    return u, expert, weight, gate


def test_gradient_of_the_block(ex):
    """E along random directions of u, the router's weights and the gate: central differences in f64, step 1e-5
    (second-order terms and rounding over the step, both near 1e-9 of the gradient's magnitudes)."""
    u, expert, weight, gate = setup(ex, drop=True)
    block = ex.ExpertBlock.random(1, 5, u.shape[1], 64)
    E, saved = block.forward(u, expert, weight, gate)
    du, dw, g = block.backward(saved)
    gen = torch.Generator("cuda").manual_seed(4)
    for name, grad in (("u", du), ("weight", dw), ("gate", g["dgate"])):
        way = torch.randn(grad.shape, dtype=torch.float64, device="cuda", generator=gen)
        h, args = 1e-5, {"u": u, "weight": weight, "gate": gate}
        e = [float(block.forward(**{**args, name: args[name] + s * h * way}, expert=expert)[0]) for s in (1, -1)]
        assert abs((e[0] - e[1]) / (2 * h) - float((grad * way).sum())) <= 1e-6 * float((grad * way).abs().sum()), name


def test_eight_bit_form_is_near(ex):
    """Ranking by 8-bit energies: a net's output is off by some parts in 100 of its size (127 steps a row, twice), so
    atomic energies, here of order 1, agree to 0.1 on average and order the atoms alike."""
    u, expert, weight, gate = setup(ex)
    block = ex.ExpertBlock.random(1, 5, u.shape[1], 64, dtype=torch.float32).quantise()
    u, weight, gate = u.float(), weight.float(), gate.float()
    e8 = block.screen(u, expert, weight, gate)
    _, saved = block.forward(u, expert, weight, gate)
    r2 = saved[8]
    e = (r2 * torch.rsqrt(r2.square().mean(1, keepdim=True) + 1e-6) * block.w2) @ block.v
    assert float((e8 - e).abs().mean()) <= 0.1 * float(e.abs().mean())
    assert float(torch.corrcoef(torch.stack([e8, e]))[0, 1]) >= 0.99


def test_example_runs(ex, capsys):
    ex.main()
    assert "8-bit" in capsys.readouterr().out
