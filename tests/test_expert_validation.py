"""The expert-block calls refuse bad arguments on the host, before any CUDA call (CPU only: the fake pointers are
never dereferenced)."""
import ctypes

import pytest
import torch

from test_call_device import OnDevice1


@pytest.fixture(scope="module")
def dpc():
    import __graft_entry__
    __graft_entry__._load_builder().build()
    import paper_2107_02103_gb300 as m
    return m


FAKE = ctypes.c_void_p(0x1000)


def test_route(dpc):
    lib = dpc._lib
    wb = dpc.dp_route_work_bytes(100000, 2, 8)
    assert wb >= 16 and lib.dp_route_work_bytes(4, 2, 8) == 1 and lib.dp_route_work_bytes(-1, 2, 8) == 0 and lib.dp_route_work_bytes(5, 65, 8) == 0
    assert lib.dp_route_work_bytes(2 ** 30, 2, 8) == 0 and lib.dp_route_work_bytes(5, 1, 1025) == 0

    def plan(expert=FAKE, ntok=100000, topk=2, nexp=8, start=FAKE, src=FAKE, pos=FAKE, work=FAKE, nbytes=wb):
        return lib.dp_route_plan(expert, ntok, topk, nexp, start, src, pos, work, nbytes, None)

    assert plan(expert=None) == plan(start=None) == plan(src=None) == plan(pos=None) == plan(work=None) == dpc.DP_ERR_NULL
    assert plan(ntok=-1) == plan(topk=0) == plan(topk=65) == plan(nexp=0) == plan(ntok=2 ** 30) == dpc.DP_ERR_SHAPE
    assert plan(nbytes=wb - 1) == plan(work=ctypes.c_void_p(0x1008)) == dpc.DP_ERR_SHAPE
    assert plan(nexp=1025) == dpc.DP_ERR_UNSUPPORTED
    for x in ("f64", "f32", "bf16", "f16"):
        gather, combine, grad = (getattr(lib, f"dp_route_{n}_{x}") for n in ("gather", "combine", "combine_grad"))
        assert gather(None, FAKE, FAKE, 4, 2, 8, FAKE, None) == dpc.DP_ERR_NULL
        assert gather(FAKE, FAKE, FAKE, 4, 2, 0, FAKE, None) == dpc.DP_ERR_SHAPE
        assert gather(ctypes.c_void_p(0x1001), FAKE, FAKE, 4, 2, 8, FAKE, None) == dpc.DP_ERR_SHAPE
        assert gather(None, None, None, 0, 2, 8, None, None) == dpc.DP_OK
        assert combine(FAKE, None, FAKE, 4, 2, 8, FAKE, None) == dpc.DP_ERR_NULL
        assert combine(FAKE, FAKE, FAKE, 4, 65, 8, FAKE, None) == dpc.DP_ERR_SHAPE
        assert grad(None, FAKE, FAKE, FAKE, FAKE, 4, 2, 8, FAKE, FAKE, None) == dpc.DP_ERR_NULL
        assert grad(FAKE, FAKE, FAKE, FAKE, FAKE, -4, 2, 8, FAKE, FAKE, None) == dpc.DP_ERR_SHAPE
        assert grad(None, None, None, None, None, 0, 2, 8, None, None, None) == dpc.DP_OK


def test_linear_i8(dpc):
    lib = dpc._lib
    odd = ctypes.c_void_p(0x1008)
    for x in ("f64", "f32", "bf16", "f16"):
        q = getattr(lib, f"dp_quant_rows_i8_{x}")
        assert q(FAKE, None, None, 4, 1, 0, FAKE, FAKE, None) == dpc.DP_ERR_SHAPE
        assert q(FAKE, None, None, 4, 2, 8, FAKE, FAKE, None) == dpc.DP_ERR_SHAPE  # topk without a plan
        assert q(FAKE, FAKE, None, 4, 2, 8, FAKE, FAKE, None) == dpc.DP_ERR_NULL
        assert q(FAKE, None, None, 4, 1, 8, odd, FAKE, None) == dpc.DP_ERR_SHAPE
        assert q(FAKE, None, None, 4, 1, 65537, FAKE, FAKE, None) == dpc.DP_ERR_UNSUPPORTED
        assert q(None, None, None, 4, 1, 8, FAKE, FAKE, None) == dpc.DP_ERR_NULL
        assert q(None, None, None, 0, 1, 8, None, None, None) == dpc.DP_OK

        def lin(xq=FAKE, rows=4, K=32, wq=FAKE, nexp=2, N=8, start=FAKE, act=0, y=FAKE, work=FAKE, nbytes=0,
                f=getattr(lib, f"dp_linear_i8_{x}")):
            return f(xq, FAKE, rows, K, wq, FAKE, None, nexp, N, start, act, y, work, nbytes, None)

        assert lin(xq=None) == lin(wq=None) == lin(y=None) == lin(start=None) == dpc.DP_ERR_NULL
        assert lin(rows=-1) == lin(K=24) == lin(K=0) == lin(N=0) == lin(nexp=0) == lin(act=2) == dpc.DP_ERR_SHAPE
        assert lin(xq=odd) == lin(wq=odd) == dpc.DP_ERR_SHAPE
        assert lin(K=65552) == dpc.DP_ERR_UNSUPPORTED
        assert lin(rows=0, xq=None, wq=None, y=None) == dpc.DP_OK
        need = lib.dp_linear_i8_work_bytes(10 ** 8, 32, 8, 2)
        assert need > 0 and lib.dp_linear_i8_work_bytes(4, 32, 8, 2) == 0
        assert lin(rows=10 ** 8, work=None, nbytes=need) == dpc.DP_ERR_NULL
        assert lin(rows=10 ** 8, nbytes=need - 1) == lin(rows=10 ** 8, work=odd, nbytes=need) == dpc.DP_ERR_SHAPE


def test_norm_gate(dpc):
    lib = dpc._lib
    wb = lib.dp_norm_gate_work_bytes(32, 4)
    assert wb > 0 and lib.dp_norm_gate_work_bytes(0, 4) == lib.dp_norm_gate_work_bytes(16385, 4) == 0
    assert lib.dp_norm_gate_work_bytes(32, 3) == 0
    for x in ("f64", "f32", "bf16", "f16"):
        def fwd(r=FAKE, gate=FAKE, gk=2, b1=FAKE, ntok=4, H=32, kind=1, eps=1e-6, u=FAKE, f=getattr(lib, f"dp_norm_gate_fwd_{x}")):
            return f(r, FAKE, gate, gk, FAKE, FAKE, b1, FAKE, FAKE, ntok, H, kind, eps, FAKE, u, FAKE, None)

        assert fwd(r=None) == fwd(gate=None) == fwd(b1=None) == fwd(u=None) == dpc.DP_ERR_NULL
        assert fwd(gk=3) == fwd(kind=2) == fwd(ntok=-1) == fwd(H=0) == fwd(eps=0.0) == dpc.DP_ERR_SHAPE
        assert fwd(H=16385) == dpc.DP_ERR_UNSUPPORTED
        assert fwd(r=ctypes.c_void_p(0x1001)) == dpc.DP_ERR_SHAPE
        assert fwd(ntok=0, r=None, gate=None, u=None) == dpc.DP_OK

        def grad(dr=FAKE, dgate=FAKE, db1=FAKE, work=FAKE, nbytes=2 * wb, kind=1, f=getattr(lib, f"dp_norm_gate_grad_{x}")):
            return f(FAKE, FAKE, FAKE, 2, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 4, 32, kind, dr, FAKE, dgate, FAKE, FAKE,
                     FAKE, db1, FAKE, work, nbytes, None)

        assert grad(dr=None) == grad(dgate=None) == grad(db1=None) == grad(work=None) == dpc.DP_ERR_NULL
        assert grad(nbytes=16) == grad(kind=-1) == grad(work=ctypes.c_void_p(0x1008)) == dpc.DP_ERR_SHAPE


def test_sizes_past_a_c_int_are_refused(dpc):
    """ctypes passes the low 32 bits of a longer size alone: a row of 2^32 + 8 elements would be one of 8."""
    big = 2 ** 32
    for bad in ((4, 2, big + 8), (4, big + 2, 8), (2 ** 64 + 4, 2, 8), (4, 2, -big + 8)):
        with pytest.raises(ValueError):
            dpc.dp_route_work_bytes(*bad)
    for bad in ((4096, big + 2048, 4096, 1), (4096, 2048, big + 4096, 1), (4096, 2048, 4096, big + 1), (2 ** 64 + 4096, 2048, 4096, 1)):
        with pytest.raises(ValueError):
            dpc.dp_linear_i8_work_bytes(*bad)
    assert dpc.dp_linear_i8_work_bytes(4096, 2048, 4096, 1) > 0
    with pytest.raises(ValueError):
        dpc.dp_norm_gate_work_bytes(big + 240, torch.float32)
    long = OnDevice1.rows(big + 8)
    with pytest.raises(ValueError, match="rows of 4294967304"):
        dpc._rows(long, "x")
    with pytest.raises(ValueError, match="4294967304 pairs"):
        dpc._pairs(long)


@pytest.mark.parametrize("x", ["f64", "f32", "bf16", "f16"])
def test_arrays_off_their_elements_are_refused(dpc, x):
    """Each array of each call in turn, one byte off: a load or store there would fault."""
    odd, lib, shape = ctypes.c_void_p(0x1001), dpc._lib, dpc.DP_ERR_SHAPE

    def each(f, args, arrays):
        for i in arrays:
            assert f(*[odd if j == i else a for j, a in enumerate(args)]) == shape, (f, i)

    n64, wb = 4, lib.dp_norm_gate_work_bytes(32, 8)
    each(lib.dp_route_plan, [FAKE, n64, 2, 8, FAKE, FAKE, FAKE, None, 0, None], (0, 4, 5, 6))
    get = lambda name: getattr(lib, f"{name}_{x}")  # noqa: E731
    each(get("dp_route_gather"), [FAKE, FAKE, FAKE, n64, 2, 8, FAKE, None], (0, 1, 2, 6))
    each(get("dp_route_combine"), [FAKE, FAKE, FAKE, n64, 2, 8, FAKE, None], (0, 1, 2, 6))
    each(get("dp_route_combine_grad"), [FAKE, FAKE, FAKE, FAKE, FAKE, n64, 2, 8, FAKE, FAKE, None], (0, 1, 2, 3, 4, 8, 9))
    each(get("dp_quant_rows_i8"), [FAKE, FAKE, FAKE, n64, 2, 8, FAKE, FAKE, None], (0, 1, 2, 6, 7))
    each(get("dp_linear_i8"), [FAKE, FAKE, n64, 32, FAKE, FAKE, FAKE, 2, 8, FAKE, 0, FAKE, None, 0, None], (0, 1, 4, 5, 6, 9, 11))
    for gate in (1, 2):
        each(get("dp_norm_gate_fwd"), [FAKE, FAKE, FAKE, gate, FAKE, FAKE, FAKE, FAKE, FAKE, n64, 32, 1, 1e-6, FAKE, FAKE, FAKE, None],
             (0, 1, 2, 4, 5, 6, 7, 8, 13, 14, 15))
        each(get("dp_norm_gate_grad"), [FAKE, FAKE, FAKE, gate] + [FAKE] * 7 + [n64, 32, 1] + [FAKE] * 9 + [wb, None],
             (0, 1, 2, *range(4, 11), *range(14, 23)))
