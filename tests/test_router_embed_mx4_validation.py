"""The router's, the embedding's and the 4-bit product's calls refuse bad arguments on the host, before any CUDA call
(CPU only: the fake pointers are never dereferenced)."""
import ctypes

import numpy as np
import pytest
import torch

from test_call_device import OnDevice1, devices, on1  # noqa: F401


@pytest.fixture(scope="module")
def dpc():
    import __graft_entry__
    __graft_entry__._load_builder().build()
    import paper_2107_02103_gb300 as m
    return m


FAKE, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1001)
ROWS = ("f64", "f32", "bf16", "f16")


@pytest.mark.parametrize("x", ROWS)
def test_route_topk(dpc, x):
    f, g = getattr(dpc._lib, f"dp_route_topk_{x}"), getattr(dpc._lib, f"dp_route_topk_grad_{x}")

    def fwd(logits=FAKE, bias=FAKE, ntok=4, nexp=8, topk=2, score=0, G=1, keep=1, top=1, renorm=1, scale=1.0, e=FAKE, w=FAKE):
        return f(logits, bias, ntok, nexp, topk, score, G, keep, top, renorm, scale, e, w, None)

    def grad(logits=FAKE, e=FAKE, dw=FAKE, ntok=4, nexp=8, topk=2, score=0, scale=1.0, dx=FAKE):
        return g(logits, e, dw, ntok, nexp, topk, score, 1, scale, dx, None)

    for kw in (dict(logits=None), dict(e=None)):
        assert fwd(**kw) == grad(**kw) == dpc.DP_ERR_NULL
    assert fwd(w=None) == grad(dw=None) == grad(dx=None) == dpc.DP_ERR_NULL
    for kw in (dict(ntok=-1), dict(nexp=0), dict(topk=0), dict(topk=9), dict(topk=65, nexp=100), dict(score=2), dict(score=-1), dict(ntok=2 ** 30),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(logits=ODD) if x != "" else {}):
        assert fwd(**kw) == grad(**kw) == dpc.DP_ERR_SHAPE, kw
    for kw in (dict(G=0), dict(G=3), dict(G=4, keep=0), dict(G=4, keep=5), dict(G=8, keep=1), dict(top=0), dict(top=3), dict(bias=ODD), dict(w=ODD), dict(e=ctypes.c_void_p(0x1002))):
        assert fwd(**kw) == dpc.DP_ERR_SHAPE, kw
    assert grad(dw=ODD) == grad(dx=ODD) == dpc.DP_ERR_SHAPE
    assert fwd(nexp=1025) == grad(nexp=1025) == dpc.DP_ERR_UNSUPPORTED
    assert f(None, None, 0, 8, 2, 0, 1, 1, 1, 1, 1.0, None, None, None) == g(None, None, None, 0, 8, 2, 0, 1, 1.0, None, None) == dpc.DP_OK
    assert fwd(ntok=0, topk=9) == dpc.DP_ERR_SHAPE


def test_embed(dpc):
    lib = dpc._lib
    assert lib.dp_embed_plan_work_bytes(100, 8) == 1 and lib.dp_embed_plan_work_bytes(0, 8) == 1
    big = 200000
    need = dpc.dp_embed_plan_work_bytes(big, 70000)
    assert need >= 16 * big
    for bad in ((-1, 8), (2 ** 31 - 4096, 8), (5, 0), (5, 2 ** 24)):
        assert lib.dp_embed_plan_work_bytes(*bad) == 0
        with pytest.raises(ValueError):
            dpc.dp_embed_plan_work_bytes(*bad)

    def plan(ids=FAKE, ntok=big, nvocab=70000, start=FAKE, src=FAKE, work=FAKE, n=need):
        return lib.dp_embed_plan(ids, ntok, nvocab, start, src, work, n, None)

    for kw in (dict(ids=None), dict(start=None), dict(src=None), dict(work=None)):
        assert plan(**kw) == dpc.DP_ERR_NULL
    for kw in (dict(ntok=-1), dict(ntok=2 ** 31 - 4096), dict(nvocab=0), dict(n=need - 1), dict(work=ctypes.c_void_p(0x1008)), dict(ids=ODD), dict(start=ctypes.c_void_p(0x1004)), dict(src=ODD)):
        assert plan(**kw) == dpc.DP_ERR_SHAPE, kw
    assert plan(nvocab=2 ** 24) == dpc.DP_ERR_UNSUPPORTED

    for bad in ((-1, 8, 4), (5, 0, 4), (5, 2 ** 20 + 1, 4), (5, 8, 3)):
        assert lib.dp_embed_grad_work_bytes(*bad) == 0
    for x, size in zip(ROWS, (8, 4, 2, 2)):
        f, g = getattr(lib, f"dp_embed_fwd_{x}"), getattr(lib, f"dp_embed_grad_{x}")
        wb = lib.dp_embed_grad_work_bytes(big, 100, size)
        assert wb > 16

        def fwd(W=FAKE, ids=FAKE, ntok=4, nvocab=8, H=100, scale=1.0, add=FAKE, y=FAKE):
            return f(W, ids, ntok, nvocab, H, scale, add, y, None)

        def grad(dy=FAKE, ids=FAKE, start=FAKE, src=FAKE, ntok=big, nvocab=8, H=100, scale=1.0, dW=FAKE, work=FAKE, n=wb):
            return g(dy, ids, start, src, ntok, nvocab, H, scale, 0, dW, work, n, None)

        for kw in (dict(W=None), dict(ids=None), dict(y=None)):
            assert fwd(**kw) == dpc.DP_ERR_NULL
        for kw in (dict(dy=None), dict(ids=None), dict(start=None), dict(src=None), dict(dW=None), dict(work=None)):
            assert grad(**kw) == dpc.DP_ERR_NULL
        for kw in (dict(ntok=-1), dict(nvocab=0), dict(H=0), dict(H=2 ** 20 + 1), dict(scale=float("nan")), dict(ids=ODD), dict(ntok=2 ** 31 - 4096)):
            assert fwd(**kw) == grad(**kw) == dpc.DP_ERR_SHAPE, kw
        assert fwd(W=ODD) == fwd(add=ODD) == fwd(y=ODD) == grad(dy=ODD) == grad(dW=ODD) == grad(n=wb - 1) == dpc.DP_ERR_SHAPE
        assert fwd(nvocab=2 ** 24) == grad(nvocab=2 ** 24) == dpc.DP_ERR_UNSUPPORTED
        assert f(None, None, 0, 8, 100, 1.0, None, None, None) == dpc.DP_OK


@pytest.mark.parametrize("x", ROWS)
def test_mx4(dpc, x):
    lib, by8 = dpc._lib, ctypes.c_void_p(0x1008)
    q, p = getattr(lib, f"dp_quant_rows_mx4_{x}"), getattr(lib, f"dp_linear_mx4_{x}")
    assert q(FAKE, None, None, 4, 1, 0, FAKE, FAKE, None) == dpc.DP_ERR_SHAPE
    assert q(FAKE, None, None, 4, 2, 8, FAKE, FAKE, None) == dpc.DP_ERR_SHAPE  # topk without a plan
    assert q(FAKE, FAKE, None, 4, 2, 8, FAKE, FAKE, None) == dpc.DP_ERR_NULL
    assert q(FAKE, None, None, 4, 1, 8, by8, FAKE, None) == dpc.DP_ERR_SHAPE
    assert q(FAKE, None, None, 4, 1, 8, FAKE, ctypes.c_void_p(0x1004), None) == dpc.DP_ERR_SHAPE
    assert q(ODD, None, None, 4, 1, 8, FAKE, FAKE, None) == dpc.DP_ERR_SHAPE
    assert q(FAKE, None, None, 4, 1, 65537, FAKE, FAKE, None) == dpc.DP_ERR_UNSUPPORTED
    assert q(None, None, None, 4, 1, 8, FAKE, FAKE, None) == dpc.DP_ERR_NULL
    assert q(None, None, None, 0, 1, 8, None, None, None) == dpc.DP_OK

    def prod(xq=FAKE, sx=FAKE, rows=300, K=128, wq=FAKE, sw=FAKE, bias=FAKE, nexp=2, N=8, start=FAKE, act=1, y=FAKE):
        return p(xq, sx, rows, K, wq, sw, bias, nexp, N, start, act, y, None)

    for kw in (dict(xq=None), dict(sx=None), dict(wq=None), dict(sw=None), dict(y=None), dict(start=None)):
        assert prod(**kw) == dpc.DP_ERR_NULL, kw
    for kw in (dict(rows=-1), dict(rows=2 ** 31 - 1), dict(K=0), dict(K=32), dict(K=96), dict(N=0), dict(N=2 ** 18 + 1), dict(nexp=0), dict(nexp=1025), dict(act=2),
               dict(xq=by8), dict(wq=by8), dict(sx=ctypes.c_void_p(0x1004)), dict(sw=ctypes.c_void_p(0x1004)), dict(bias=ODD), dict(start=ctypes.c_void_p(0x1004)), dict(y=ODD)):
        assert prod(**kw) == dpc.DP_ERR_SHAPE, kw
    assert prod(K=65600) == dpc.DP_ERR_UNSUPPORTED
    assert p(None, None, 0, 64, None, None, None, 1, 8, None, 0, None, None) == dpc.DP_OK


def test_binding(dpc):
    """The Python calls check types and shapes before the library is called."""
    x, i32 = on1(4, 8), on1(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        dpc.dp_route_topk(x, 2, score="relu")
    with pytest.raises(ValueError):
        dpc.dp_route_topk(x, 2, bias=on1(7))
    with pytest.raises(TypeError):
        dpc.dp_route_topk(x.to(torch.int32), 2)
    with pytest.raises(TypeError):
        dpc.dp_route_topk(torch.zeros(4, 8), 2)  # on the CPU
    with pytest.raises(ValueError):
        dpc.dp_route_topk(on1(8, 4).t(), 2)  # strided
    with pytest.raises(TypeError):
        dpc.dp_route_topk_grad(x, on1(4, 2, dtype=torch.int64), on1(4, 2))
    with pytest.raises(ValueError):
        dpc.dp_route_topk_grad(x, on1(3, 2, dtype=torch.int32), on1(4, 2))
    with pytest.raises(ValueError):
        dpc.dp_route_topk(x, 2 ** 40)
    with pytest.raises(TypeError):
        dpc.dp_embed_fwd(x, i32.to(torch.int64))
    with pytest.raises(ValueError):
        dpc.dp_embed_fwd(x, i32, add=on1(4, 9))
    with pytest.raises(ValueError):
        dpc.dp_embed_grad(x, i32, on1(6, dtype=torch.int64), i32, accumulate=True)
    with pytest.raises(ValueError):
        dpc.dp_embed_grad(x, i32, on1(1, dtype=torch.int64), i32)
    with pytest.raises(ValueError):
        dpc.dp_quant_rows_mx4(x, src=i32)
    q, s = on1(4, 64, dtype=torch.uint8), on1(4, 8, dtype=torch.uint8)
    with pytest.raises(ValueError):
        dpc.dp_linear_mx4(q, s, on1(1, 3, 32, dtype=torch.uint8), on1(1, 3, 8, dtype=torch.uint8))
    with pytest.raises(ValueError):
        dpc.dp_linear_mx4(q, on1(4, 4, dtype=torch.uint8), on1(1, 3, 64, dtype=torch.uint8), on1(1, 3, 8, dtype=torch.uint8))
    with pytest.raises(ValueError):
        dpc.dp_linear_mx4(q, s, on1(1, 3, 64, dtype=torch.uint8), on1(1, 3, 8, dtype=torch.uint8), act="relu")
    with pytest.raises(TypeError):
        dpc.dp_linear_mx4(q.to(torch.int8), s, on1(1, 3, 64, dtype=torch.uint8), on1(1, 3, 8, dtype=torch.uint8))
    wide = OnDevice1.rows(2 ** 31)
    with pytest.raises(ValueError):
        dpc.dp_route_topk(wide, 2)


def test_reference_quantiser():
    """The tests' own quantiser on values worked out by hand."""
    import mx4_common as M
    x = np.zeros((1, 70))
    x[0, :8] = [6.0, -0.25, 0.75, 2.5, -5.0, 7.9, 0.2, -0.0]
    x[0, 64] = 3.0
    code, scale = M.quantise(x)
    assert list(code[0, :8]) == [7, 8, 2, 4, 14, 7, 0, 8] and code.shape == (1, 128)
    assert list(scale[0]) == [127, 0, 126, 0, 0, 0, 0, 0]
    v = M.values(M.pack(code), scale)
    assert list(v[0, :6]) == [6.0, 0.0, 1.0, 2.0, -4.0, 6.0] and v[0, 64] == 3.0


def calls(dpc):
    i32, i64, u8 = torch.int32, torch.int64, torch.uint8
    x, w, e, ids = on1(4, 32), on1(4, 2), on1(4, 2, dtype=i32), on1(4, dtype=i32)
    q, s = on1(4, 32, dtype=u8), on1(4, 8, dtype=u8)
    plan, work = (on1(9, dtype=i64), ids), on1(1 << 16, dtype=u8)
    return {
        "dp_route_topk_f32": lambda: dpc.dp_route_topk(x, 2, out=(e, w)),
        "dp_route_topk_grad_f32": lambda: dpc.dp_route_topk_grad(x, e, w, out=x),
        "dp_quant_rows_mx4_f32": lambda: dpc.dp_quant_rows_mx4(x, out=(q, s)),
        "dp_linear_mx4_f32": lambda: dpc.dp_linear_mx4(q, s, q[None], s[None], out=on1(4, 4)),
        "dp_embed_plan": lambda: dpc.dp_embed_plan(ids, 8, out=plan),
        "dp_embed_fwd_f32": lambda: dpc.dp_embed_fwd(on1(8, 32), ids, add=x, out=x),
        "dp_embed_grad_f32": lambda: dpc.dp_embed_grad(x, ids, *plan, out=on1(8, 32), work=work),
    }


@pytest.mark.parametrize("name", ["dp_route_topk_f32", "dp_route_topk_grad_f32", "dp_quant_rows_mx4_f32", "dp_linear_mx4_f32", "dp_embed_plan",
                                  "dp_embed_fwd_f32", "dp_embed_grad_f32"])
@pytest.mark.parametrize("current", [0, 1])
def test_launches_on_the_tensors_device(dpc, devices, monkeypatch, name, current):  # noqa: F811
    devices[0] = current
    seen = []
    real = getattr(dpc._lib, name)

    def launch(*args):
        assert len(args) == len(real.argtypes)
        seen.append((devices[0], getattr(args[-1], "value", args[-1])))
        return 0

    monkeypatch.setattr(dpc._lib, name, launch)
    for table in dpc._ROW_FN.values():
        for t, fn in table.items():
            if fn is real:
                monkeypatch.setitem(table, t, launch)
    calls(dpc)[name]()
    assert seen == [(1, 101)] and devices[0] == current
