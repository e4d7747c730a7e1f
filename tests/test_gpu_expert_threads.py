"""Calls of different sizes from several host threads at once, each on its own stream: a kernel's shared-memory limit
is shared by them all, so no call may set it to its own size.  The loops run in C, where nothing serialises them."""
import ctypes
import subprocess
import threading

import pytest
import torch

from gpu_common import lib, need_gpu

pytestmark = pytest.mark.gpu

LOOPS = """
#include <stddef.h>
#include <stdint.h>
typedef int plan_fn(const int32_t *, int64_t, int, int, int64_t *, int32_t *, int32_t *, void *, size_t, void *);
int plan_loop(int n, plan_fn *f, const int32_t *e, int64_t ntok, int topk, int nexp, int64_t *start, int32_t *src,
              int32_t *pos, void *stream) {
  for (int rc; n > 0; --n)
    if ((rc = f(e, ntok, topk, nexp, start, src, pos, NULL, 0, stream))) return rc;
  return 0;
}
typedef int desc_fn(const void *, int64_t, int, int, void *, void *);
int desc_loop(int n, desc_fn *f, const void *T, int64_t nloc, int M1, int M2, void *D, void *stream) {
  for (int rc; n > 0; --n)
    if ((rc = f(T, nloc, M1, M2, D, stream))) return rc;
  return 0;
}
typedef int norm_fn(const void *, const void *, const void *, int, const void *, const void *, const void *,
                    const void *, const void *, int64_t, int, int, double, void *, void *, void *, void *);
int norm_loop(int n, norm_fn *f, const void *x, const void *v, int64_t ntok, int H, void *r2, void *u, void *stats,
              void *stream) {
  for (int rc; n > 0; --n)
    if ((rc = f(x, x, NULL, 0, v, v, NULL, v, NULL, ntok, H, 0, 1e-6, r2, u, stats, stream))) return rc;
  return 0;
}
"""


@pytest.fixture(scope="module")
def loops(tmp_path_factory):
    need_gpu()
    d = tmp_path_factory.mktemp("loops")
    (d / "loops.c").write_text(LOOPS)
    subprocess.run(["gcc", "-std=c99", "-O1", "-shared", "-fPIC", str(d / "loops.c"), "-o", str(d / "loops.so")], check=True)
    return ctypes.CDLL(str(d / "loops.so"))


def at_once(work):
    """Each function called with a stream of its own in a thread of its own; their results."""
    go, rc = threading.Barrier(len(work)), [None] * len(work)
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()

    def one(i):
        go.wait(60)
        rc[i] = work[i](ctypes.c_void_p(streams[i].cuda_stream))

    threads = [threading.Thread(target=one, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return rc


def ptr(t):
    return ctypes.c_void_p(t.data_ptr())


def test_plans_of_few_and_many_experts(loops):
    dpc = lib()
    cases = []
    for nexp in (400, 1024, 500, 1000):
        expert = (torch.arange(96, dtype=torch.int32, device="cuda").view(48, 2) * 7 % nexp).contiguous()
        cases.append((expert, nexp, dpc.dp_route_plan(expert, nexp), tuple(torch.empty_like(t) for t in dpc.dp_route_plan(expert, nexp))))
    work = [lambda s, e=e, n=n, o=o: loops.plan_loop(20000, dpc._lib.dp_route_plan, ptr(e), ctypes.c_int64(48), 2, n, *map(ptr, o), s)
            for e, n, _, o in cases]
    assert at_once(work) == [0] * len(work)
    for _, _, ref, got in cases:
        assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_norms_of_short_and_long_rows(loops):
    dpc = lib()
    cases = []
    for H in (2048, 1600, 1284, 1928):
        x, v = torch.randn(4, H, device="cuda"), torch.ones(H, device="cuda")
        ref = dpc.dp_norm_gate_fwd(x, x, v, v, v)
        cases.append((x, v, H, ref, tuple(torch.empty_like(t) for t in ref)))
    work = [lambda s, x=x, v=v, H=H, o=o: loops.norm_loop(20000, dpc._lib.dp_norm_gate_fwd_f32, ptr(x), ptr(v), ctypes.c_int64(4),
                                                          H, *map(ptr, o), s) for x, v, H, _, o in cases]
    assert at_once(work) == [0] * len(work)
    for *_, ref, got in cases:
        assert all(torch.equal(a, b) for a, b in zip(ref, got))


def test_descriptors_of_short_and_long_rows(loops):
    dpc = lib()
    cases = []
    for M1 in (512, 1000, 600, 1600):
        T = torch.randn(4, 4, M1, dtype=torch.float64, device="cuda")
        ref = dpc.dp_descriptor_contract(T, 2)
        cases.append((T, M1, ref, torch.empty_like(ref)))
    work = [lambda s, T=T, M1=M1, D=D: loops.desc_loop(20000, dpc._lib.dp_descriptor_contract_f64, ptr(T), ctypes.c_int64(4), M1, 2,
                                                       ptr(D), s) for T, M1, _, D in cases]
    assert at_once(work) == [0] * len(work)
    for _, _, ref, got in cases:
        assert torch.equal(ref, got)
