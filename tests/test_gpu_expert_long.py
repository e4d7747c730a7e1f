"""Arrays past 2^31 elements (4.5 GB each) through the expert-block calls: the last rows equal those of a call on
them alone."""
import pytest
import torch

from gpu_common import lib, need_gpu

pytestmark = [pytest.mark.gpu, pytest.mark.slow]
T, H, TAIL = 1_100_003, 2048, 97
BF = torch.bfloat16


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    yield
    torch.cuda.empty_cache()


def big(seed):
    g = torch.Generator("cuda").manual_seed(seed)
    t = torch.empty(T, H, dtype=BF, device="cuda")
    t.normal_(generator=g)
    return t


def test_norm():
    dpc = lib()
    r, f = big(1), big(2)
    a, w1, w2 = (torch.rand(H, device="cuda") for _ in range(3))
    r2, u, st = dpc.dp_norm_gate_fwd(r, f, a, w1, w2)
    r2t, ut, stt = dpc.dp_norm_gate_fwd(r[-TAIL:].contiguous(), f[-TAIL:].contiguous(), a, w1, w2)
    assert torch.equal(r2[-TAIL:], r2t) and torch.equal(u[-TAIL:], ut) and torch.equal(st[-TAIL:], stt)
    g = dpc.dp_norm_gate_grad(r2, f, a, w1, w2, st, r, u)
    gt = dpc.dp_norm_gate_grad(r2t, f[-TAIL:].contiguous(), a, w1, w2, stt, r[-TAIL:].contiguous(), ut)
    assert torch.equal(g["dr"][-TAIL:], gt["dr"]) and torch.equal(g["df"][-TAIL:], gt["df"])


def test_route():
    dpc = lib()
    x = big(3)
    expert = (torch.arange(T, device="cuda", dtype=torch.int32) % 3).view(T, 1)
    start, src, pos = dpc.dp_route_plan(expert, 3)
    xs = dpc.dp_route_gather(x, src, pos)
    assert torch.equal(xs[-TAIL:], x[src[-TAIL:].long()]) and torch.equal(xs[:TAIL], x[src[:TAIL].long()])
    w = torch.rand(T, 1, device="cuda")
    y = dpc.dp_route_combine(xs, pos, w)
    assert torch.equal(y[-TAIL:], (x[-TAIL:].float() * w[-TAIL:]).to(BF))
    dz, dw = dpc.dp_route_combine_grad(xs, src, pos, w, x)
    assert torch.equal(dz[-TAIL:], (x[src[-TAIL:].long()].float() * w[src[-TAIL:].long()]).to(BF))
    assert torch.allclose(dw[-TAIL:, 0], x[-TAIL:].float().square().sum(1), rtol=1e-5)


def test_integers_and_product():
    dpc = lib()
    x = big(4)
    xq, sx = dpc.dp_quant_rows_i8(x)
    xt, st = dpc.dp_quant_rows_i8(x[-TAIL:].contiguous())
    assert torch.equal(xq[-TAIL:], xt) and torch.equal(sx[-TAIL:], st)
    del x
    wq = torch.randint(-127, 128, (1, H, H), dtype=torch.int8, device="cuda")
    sw = torch.rand(1, H, device="cuda") * 1e-3
    y = dpc.dp_linear_i8(xq, sx, wq, sw, dtype=BF)
    assert torch.equal(y[-TAIL:], dpc.dp_linear_i8(xt, st, wq, sw, dtype=BF))
    assert torch.equal(y[:5], dpc.dp_linear_i8(xq[:5].contiguous(), sx[:5].contiguous(), wq, sw, dtype=BF))
