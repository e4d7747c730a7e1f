"""The norms on many whole rows: enough of them that every block goes round its stages several times, every row and
every column sum against 64 bits (torch on the GPU), with bounds of the kernels' arithmetic."""
import pytest
import torch

from gpu_common import lib, need_gpu
from rows_common import SUM_UNIT, TINY, UNIT, wtype

pytestmark = pytest.mark.gpu
EPS = 1e-6
D = torch.float64


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def near(got, ref, bound, what):
    over = (got.double() - ref).abs() - bound
    assert got.shape == ref.shape and bool((over <= 0).all()), f"{what}: beyond its bound by {float(over.nan_to_num(torch.inf).max()):.3e}"


def top(v):
    return v.abs().amax(1, keepdim=True)


def inputs(T, H, dtype, kind, gate):
    g = torch.Generator("cuda").manual_seed(T + H)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=D)  # noqa: E731
    t = {n: (rn(T, H) * (3.0 if n == "f" else 1.0) + (0.5 if n == "f" else 0.0)).to(dtype) for n in ("r", "f", "dr2", "du")}
    t["gate"] = None if gate == "none" else (rn(*((T, H) if gate == "full" else (T,))) * 0.5 + 0.5).to(dtype)
    for n, c in (("a", 0.1), ("w1", 1.0), ("w2", 1.0), ("b1", 0.0), ("b2", 0.0)):
        t[n] = (rn(H) * 0.1 + c).to(wtype(dtype)) if kind == "layer" or n[0] != "b" else None
    d = {n: torch.zeros((), dtype=D, device="cuda") if x is None else x.double() for n, x in t.items()}
    d["gate"] = torch.ones(T, 1, dtype=D, device="cuda") if gate == "none" else d["gate"].reshape(T, -1)
    return t, d


def normed(v, kind):
    m = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    return m, ((v - m).square().mean(1, keepdim=True) + EPS).rsqrt()


CASES = [(60001, 240), (20003, 512), (20003, 1600), (20005, 1792), (20003, 2048), (7001, 4096), (5003, 6000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16, torch.float64], ids=["f32", "bf16", "f16", "f64"])
@pytest.mark.parametrize("T,H", CASES)
@pytest.mark.parametrize("kind,gate", [("rms", "full"), ("layer", "full"), ("layer", "token"), ("rms", "none")])
def test_all_rows_and_sums(dtype, T, H, kind, gate):
    """Bounds: a row's sums pass at most 64 additions from element to total, so a mean is off by 64 units of the largest
    magnitude and s by 40 relative, with the epilogue's handful below 128 units of (1 + |value|) times the row's largest
    normed magnitude, and one rounding to the row type (twice that for the backward's means of normed terms).  Column
    sums: that of their terms, and the additions of a block's rows and of the partials on their sum."""
    dpc = lib()
    t, d = inputs(T, H, dtype, kind, gate)
    layer, G = kind == "layer", d["gate"]
    r2, u, st = dpc.dp_norm_gate_fwd(*(t[n] for n in ("r", "f", "a", "w1", "w2", "b1", "b2", "gate")), kind, EPS)
    a, un, tiny = 128 * SUM_UNIT[dtype], UNIT[dtype], TINY[dtype]
    m1, s1 = normed(d["f"], kind)
    rr = d["r"] + d["a"] * G * ((d["f"] - m1) * s1 * d["w1"] + d["b1"])
    m2, s2 = normed(rr, kind)
    ru = (rr - m2) * s2 * d["w2"] + d["b2"]
    mag, mag2 = 1 + top(d["f"]) * s1, 1 + top(rr) * s2
    near(r2, rr, un * rr.abs() + a * (1 + top(rr)) * mag + tiny, "r2")
    near(u, ru, un * ru.abs() + a * (1 + top(ru)) * mag * mag2 + tiny, "u")
    near(st, torch.cat([m1, s1, m2, s2], 1), a * torch.cat([1 + top(d["f"]), s1 * mag ** 2, (1 + top(rr)) * mag, s2 * (mag * mag2) ** 2], 1), "stats")
    del rr, ru

    got = dpc.dp_norm_gate_grad(r2, *(t[n] for n in ("f", "a", "w1", "w2")), st, t["dr2"], t["du"], t["b1"], t["b2"], t["gate"], kind)
    m1, s1, m2, s2 = st.double().split(1, 1)
    mean = (lambda v: v.mean(1, keepdim=True)) if layer else (lambda v: 0.0)
    n1, n2 = (d["f"] - m1) * s1, (r2.double() - m2) * s2
    v = d["du"] * d["w2"]
    dr = d["dr2"] + s2 * (v - n2 * (v * n2).mean(1, keepdim=True) - mean(v))
    p = n1 * d["w1"] + d["b1"]
    dp = dr * d["a"] * G
    v = dp * d["w1"]
    df = s1 * (v - n1 * (v * n1).mean(1, keepdim=True) - mean(v))
    dr_mag = top(d["dr2"]) + s2 * top(d["du"] * d["w2"]) * (1 + top(n2) ** 2)
    near(got["dr"], dr, un * dr.abs() + 2 * a * dr_mag + tiny, "dr")
    df_mag = s1 * top(dr_mag * (d["a"] * d["w1"]).abs() * G.abs()) * (1 + top(n1) ** 2)
    near(got["df"], df, un * df.abs() + 4 * a * df_mag + tiny, "df")
    if gate != "none":
        dg, dg_mag = dr * d["a"] * p, dr_mag * d["a"].abs() * (p.abs() + d["b1"].abs() + n1.abs())
        if gate == "token":
            dg, dg_mag = dg.sum(1), dg_mag.sum(1)
        near(got["dgate"], dg, un * dg.abs() + 4 * a * dg_mag + tiny, "dgate")
    cols = {"da": (dr * G * p, dr_mag * G.abs() * (p.abs() + d["b1"].abs())), "dw1": (dp * n1, dr_mag * d["a"].abs() * G.abs() * (n1.abs() + 1e-3)),
            "dw2": (d["du"] * n2, d["du"].abs() * (n2.abs() + 1e-3))}
    if layer:
        cols.update(db1=(dp, dr_mag * d["a"].abs() * G.abs()), db2=(d["du"], d["du"].abs()))
    for n, (c, m) in cols.items():
        near(got[n], c.sum(0), (4 * a + (T // 152 + 64) * SUM_UNIT[dtype]) * m.sum(0), n)
