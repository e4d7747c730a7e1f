"""Arrays past 2^31 elements: the last rows are those of a call on them alone, bit for bit."""
import pytest
import torch

from gpu_common import lib, need_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()
    yield
    torch.cuda.empty_cache()


def test_router():
    dpc = lib()
    T, E, k = 2_200_003, 1000, 8
    x = torch.empty(T, E, dtype=torch.bfloat16, device="cuda").normal_()
    b = 0.01 * torch.randn(E, device="cuda")
    kw = dict(bias=b, score="sigmoid", ngroup=10, keep_groups=4)
    e, w = dpc.dp_route_topk(x, k, **kw)
    dw = torch.randn(T, k, device="cuda")
    tail = slice(T - 1000, T)
    e1, w1 = dpc.dp_route_topk(x[tail].contiguous(), k, **kw)
    assert torch.equal(e[tail], e1) and torch.equal(w[tail], w1)
    for renorm, score in ((True, "sigmoid"), (False, "softmax")):
        dx = dpc.dp_route_topk_grad(x, e, dw, score=score, renorm=renorm)
        d1 = dpc.dp_route_topk_grad(x[tail].contiguous(), e1, dw[tail].contiguous(), score=score, renorm=renorm)
        assert torch.equal(dx[tail], d1)
        del dx


def test_embedding():
    """A long table, many rows, and a gradient whose rows and sums lie past 2^31."""
    dpc = lib()
    V = T = 2_200_001
    H = 1000
    W = torch.empty(V, H, dtype=torch.float16, device="cuda").normal_()
    ids = torch.arange(T - 1, -1, -1, dtype=torch.int32, device="cuda")
    y = dpc.dp_embed_fwd(W, ids, add=W)
    assert torch.equal(y[:50], (W[:50].float() + W.flip(0)[:50].float()).half()) and torch.equal(y[-50:], y.flip(0)[-50:])
    start, src = dpc.dp_embed_plan(ids, V)
    assert torch.equal(src, ids) and torch.equal(start, torch.arange(V + 1, device="cuda"))
    dW = dpc.dp_embed_grad(y, ids, start, src, scale=0.5)
    assert torch.equal(dW[-77:], 0.5 * y.flip(0)[-77:].float()) and torch.equal(dW[:77], 0.5 * y.flip(0)[:77].float())


@pytest.mark.parametrize("N", [8, 1000])
def test_four_bit_product(N):
    dpc = lib()
    n, K = 2_300_001, 2048
    x = torch.empty(n, K, dtype=torch.bfloat16, device="cuda").normal_()
    xq, sx = dpc.dp_quant_rows_mx4(x)
    tail = slice(n - 500, n)
    q1, s1 = dpc.dp_quant_rows_mx4(x[tail].contiguous())
    assert torch.equal(xq[tail], q1) and torch.equal(sx[tail], s1)
    del x
    wq, sw = dpc.dp_quant_rows_mx4(torch.randn(N, K, device="cuda"))
    y = dpc.dp_linear_mx4(xq, sx, wq[None], sw[None], dtype=torch.bfloat16)
    # one tile's sums do not depend on its other rows
    assert torch.equal(y[tail], dpc.dp_linear_mx4(q1, s1, wq[None], sw[None], dtype=torch.bfloat16))
    assert dpc.dp_tc_wait_timeouts() == 0
