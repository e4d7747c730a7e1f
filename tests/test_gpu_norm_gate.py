"""The norms around a block with gate and residual scale on the GPU, forward and backward, against 64 bits with
bounds of their arithmetic, and the backward against central differences."""
import numpy as np
import pytest
import torch

from gpu_common import lib, need_gpu
from rows_common import IDS, ROWS, SUM_UNIT, TINY, UNIT, f64, offset_view, rnd, within, wtype

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(autouse=True)
def _gpu():
    need_gpu()


def inputs(seed, T, H, dtype, kind, gate, shift=0.5):
    wd = wtype(dtype)
    d = {}
    for i, (name, shape, scale, mean, t) in enumerate((
            ("r", (T, H), 1.0, 0.0, dtype), ("f", (T, H), 3.0, shift, dtype), ("a", (H,), 0.02, 0.1, wd),
            ("w1", (H,), 0.1, 1.0, wd), ("w2", (H,), 0.1, 1.0, wd), ("b1", (H,), 0.1, 0.0, wd), ("b2", (H,), 0.1, 0.0, wd),
            ("gate", (T, H) if gate == "full" else (T,), 0.5, 0.5, dtype), ("dr2", (T, H), 1.0, 0.0, dtype),
            ("du", (T, H), 1.0, 0.0, dtype))):
        d[name] = rnd(seed * 16 + i, *shape, dtype=t, scale=scale, shift=mean)
    if gate == "none":
        d["gate"] = (None, np.ones(1))
    if kind == "rms":
        d["b1"] = d["b2"] = (None, np.zeros(H))
    return d


def normed(v, kind):
    m = v.mean(1, keepdims=True) if kind == "layer" else np.zeros((v.shape[0], 1))
    return m, 1.0 / np.sqrt(((v - m) ** 2).mean(1, keepdims=True) + EPS)


def forward(d, kind):
    g = d["gate"][1]
    g = g[:, None] if g.ndim == 1 and g.size != 1 else g
    m1, s1 = normed(d["f"][1], kind)
    p = (d["f"][1] - m1) * s1 * d["w1"][1] + d["b1"][1]
    r2 = d["r"][1] + d["a"][1] * (g.reshape(-1, 1) if g.ndim == 1 else g) * p
    m2, s2 = normed(r2, kind)
    return r2, (r2 - m2) * s2 * d["w2"][1] + d["b2"][1], np.concatenate([m1, s1, m2, s2], 1)


SHAPES = [(1, 1), (1, 240), (3, 7), (5, 256), (4, 257), (33, 1003), (40, 1600), (9, 2048), (2, 4099), (3, 8192), (2, 9000),
          (2, 16384), (0, 64), (700, 36), (2003, 259), (1500, 1003), (1301, 512), (999, 2041), (1300, 1530)]


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,H", SHAPES)
@pytest.mark.parametrize("kind,gate,offset", [("rms", "full", 0), ("layer", "full", 1), ("layer", "token", 0),
                                              ("rms", "none", 1)])
def test_forward(dtype, T, H, kind, gate, offset):
    """Bounds: a row's sums pass at most 64 additions from element to total, so the mean is off by 64 units of
    the largest magnitude and s by 40 relative; with the epilogue's handful that is below 128 units of
    (1 + |value|) times the row's largest normed magnitude; one rounding to the row type on top."""
    dpc = lib()
    d = inputs(T + H, T, H, dtype, kind, gate)
    g = lambda n: offset_view(d[n][0]) if offset and d[n][0] is not None and d[n][0].dim() == 2 else d[n][0]  # noqa: E731
    r2, u, stats = dpc.dp_norm_gate_fwd(g("r"), g("f"), g("a"), g("w1"), g("w2"), g("b1"), g("b2"), g("gate"), kind, EPS)
    rr, ru, rst = forward(d, kind)
    if T == 0:
        return
    a, t = 128 * SUM_UNIT[dtype], UNIT[dtype]
    big = lambda v: 1 + np.abs(v).max(1, keepdims=True)  # noqa: E731
    mag = 1 + np.abs(d["f"][1]).max(1, keepdims=True) * rst[:, 1:2]  # normed magnitude before the mean comes off
    within(r2, rr, t * np.abs(rr) + a * big(rr) * mag + TINY[dtype], "r2")
    mag2 = 1 + np.abs(rr).max(1, keepdims=True) * rst[:, 3:4]
    # a row of one element has r2^ = 0 or +-1: the layer norm's difference cancels to nothing there
    within(u, ru, t * np.abs(ru) + a * big(ru) * mag * mag2 + TINY[dtype], "u")
    scale = np.concatenate([big(d["f"][1]), rst[:, 1:2] * mag ** 2, big(rr) * mag, rst[:, 3:4] * (mag * mag2) ** 2], 1)
    within(stats, rst, a * scale, "stats")


def backward(d, r2, stats, kind, gate):
    m1, s1, m2, s2 = (stats[:, i:i + 1] for i in range(4))
    f, du, a = d["f"][1], d["du"][1], d["a"][1]
    G = d["gate"][1]
    G = np.ones((f.shape[0], 1)) if gate == "none" else G[:, None] if gate == "token" else G
    n1, n2 = (f - m1) * s1, (r2 - m2) * s2
    mean = (lambda v: v.mean(1, keepdims=True)) if kind == "layer" else (lambda v: 0.0)
    t = du * d["w2"][1]
    dr = d["dr2"][1] + s2 * (t - n2 * (t * n2).mean(1, keepdims=True) - mean(t))
    p = n1 * d["w1"][1] + d["b1"][1]
    dp = dr * a * G
    t1 = dp * d["w1"][1]
    df = s1 * (t1 - n1 * (t1 * n1).mean(1, keepdims=True) - mean(t1))
    dg = dr * a * p
    rows = {"dr": dr, "df": df, "dgate": dg if gate == "full" else dg.sum(1) if gate == "token" else None}
    cols = {"da": dr * G * p, "dw1": dp * n1, "dw2": du * n2}
    if kind == "layer":
        cols.update(db1=dp, db2=du)
    return rows, cols, (s1, s2, n1, n2, p, dg)


@pytest.mark.parametrize("dtype", ROWS, ids=IDS)
@pytest.mark.parametrize("T,H", SHAPES)
@pytest.mark.parametrize("kind,gate,offset", [("rms", "full", 0), ("layer", "full", 1), ("layer", "token", 0),
                                              ("rms", "none", 1)])
def test_backward(dtype, T, H, kind, gate, offset):
    """The reference takes the same rounded r2 and stats.  Row results: 256 units of the row's largest term
    (means of 64-addition sums times normed values); column sums: 256 units of the terms' magnitudes for the
    terms themselves, and the additions of a thread's rows and of the partials, T + 64, on their sum."""
    dpc = lib()
    d = inputs(3 * T + H, T, H, dtype, kind, gate)
    fr2, _, fst = forward(d, kind)
    r2, stats = torch.from_numpy(fr2).to(dtype).cuda(), torch.from_numpy(fst).to(wtype(dtype)).cuda()
    if T:
        rows, cols, (s1, s2, n1, n2, p, dg) = backward(d, f64(r2), f64(stats), kind, gate)
    g = lambda n: offset_view(d[n][0]) if offset and d[n][0] is not None and d[n][0].dim() == 2 else d[n][0]  # noqa: E731
    got = dpc.dp_norm_gate_grad(offset_view(r2) if offset else r2, g("f"), g("a"), g("w1"), g("w2"), stats, g("dr2"),
                                g("du"), g("b1"), g("b2"), g("gate"), kind)
    names = ["da", "dw1", "dw2"] + (["db1", "db2"] if kind == "layer" else [])
    assert {k for k, v in got.items() if v is not None} == {"dr", "df", *names} | (set() if gate == "none" else {"dgate"})
    if T == 0:
        assert not any(got[n].any() for n in names)
        return
    a, t = 256 * SUM_UNIT[dtype], UNIT[dtype]
    top = lambda v: np.abs(v).max(1, keepdims=True)  # noqa: E731
    m2 = 1 + top(n2) ** 2
    dr_mag = (top(d["dr2"][1]) + s2 * top(d["du"][1] * d["w2"][1]) * m2) * np.ones((1, H))
    within(got["dr"], rows["dr"], t * np.abs(rows["dr"]) + a * dr_mag + TINY[dtype], "dr")
    G = 1.0 if gate == "none" else np.abs(d["gate"][1]).reshape(T, -1)
    t1_mag = top(dr_mag * np.abs(d["a"][1] * d["w1"][1]) * G)
    df_mag = s1 * t1_mag * (1 + top(n1) ** 2)
    within(got["df"], rows["df"], t * np.abs(rows["df"]) + 2 * a * df_mag + TINY[dtype], "df")
    dg_mag = dr_mag * np.abs(d["a"][1]) * (np.abs(p) + np.abs(d["b1"][1]) + np.abs(n1))
    if gate == "full":
        within(got["dgate"], rows["dgate"], t * np.abs(rows["dgate"]) + 2 * a * dg_mag + TINY[dtype], "dgate")
    elif gate == "token":
        within(got["dgate"], rows["dgate"], t * np.abs(rows["dgate"]) + 2 * a * dg_mag.sum(1) + TINY[dtype], "dgate")
    mags = {"da": dr_mag * G * (np.abs(p) + np.abs(d["b1"][1])), "dw1": dr_mag * np.abs(d["a"][1]) * G * (np.abs(n1) + 1e-3),
            "dw2": np.abs(d["du"][1]) * (np.abs(n2) + 1e-3), "db1": dr_mag * np.abs(d["a"][1]) * G, "db2": np.abs(d["du"][1])}
    for n in names:
        within(got[n], cols[n].sum(0), (2 * a + (T + 64) * SUM_UNIT[dtype]) * mags[n].sum(0) + 1e-300, n)


@pytest.mark.parametrize("kind,gate", [("rms", "full"), ("layer", "full"), ("layer", "token"), ("rms", "none")])
def test_backward_against_differences(kind, gate):
    """E = <dr2, r2> + <du, u> along a random direction of every input, central differences in f64 (step 1e-5:
    h^2 times third derivatives and rounding over h, both about 1e-10 of the gradient's magnitudes)."""
    dpc = lib()
    T, H = 6, 300
    d = inputs(5, T, H, torch.float64, kind, gate)
    names = [n for n in ("r", "f", "a", "w1", "w2", "b1", "b2", "gate") if d[n][0] is not None]
    way = {n: rnd(900 + i, *d[n][0].shape)[0] for i, n in enumerate(names)}

    def energy(h):
        v = {n: (d[n][0] + h * way[n] if n in way else None) for n in ("r", "f", "a", "w1", "w2", "b1", "b2", "gate")}
        r2, u, st = dpc.dp_norm_gate_fwd(v["r"], v["f"], v["a"], v["w1"], v["w2"], v["b1"], v["b2"], v["gate"], kind, EPS)
        return float((d["dr2"][0] * r2).sum() + (d["du"][0] * u).sum()), r2, st

    _, r2, st = energy(0.0)
    g = dpc.dp_norm_gate_grad(r2, *(d[n][0] for n in ("f", "a", "w1", "w2")), st, d["dr2"][0], d["du"][0], d["b1"][0],
                              d["b2"][0], d["gate"][0], kind)
    terms = [(f64(g["d" + n]) * f64(way[n])).ravel() for n in names]
    h = 1e-5
    num = (energy(h)[0] - energy(-h)[0]) / (2 * h)
    assert abs(num - sum(t.sum() for t in terms)) <= 1e-7 * sum(np.abs(t).sum() for t in terms)


def test_special_rows():
    """Zero rows give finite results (eps); a NaN or infinity stays in its row."""
    dpc = lib()
    d = inputs(1, 8, 500, torch.float32, "rms", "full")
    r, f = d["r"][0].clone(), d["f"][0].clone()
    clean = dpc.dp_norm_gate_fwd(r, f, d["a"][0], d["w1"][0], d["w2"][0], gate=d["gate"][0])
    f[2] = 0
    r[3], f[3] = 0, 0
    f[5, 7] = float("nan")
    r[6, 0] = float("inf")
    r2, u, _ = dpc.dp_norm_gate_fwd(r, f, d["a"][0], d["w1"][0], d["w2"][0], gate=d["gate"][0])
    assert torch.equal(r2[2], r[2]) and not u[3].any() and not r2[3].any()
    assert torch.isnan(u[5]).all() and torch.isnan(u[6]).any()
    for i in (0, 1, 4, 7):
        assert torch.equal(r2[i], clean[0][i]) and torch.equal(u[i], clean[1][i])


def test_repeats_bit_for_bit():
    dpc = lib()
    d = inputs(2, 3000, 1600, torch.float32, "layer", "full")
    r2, u, st = dpc.dp_norm_gate_fwd(*(d[n][0] for n in ("r", "f", "a", "w1", "w2", "b1", "b2", "gate")), kind="layer")
    run = lambda: dpc.dp_norm_gate_grad(r2, *(d[n][0] for n in ("f", "a", "w1", "w2")), st, d["dr2"][0], d["du"][0],  # noqa: E731
                                        d["b1"][0], d["b2"][0], d["gate"][0], "layer")
    a, b = run(), run()
    assert all(torch.equal(a[k], b[k]) for k in a)


def test_refusals():
    dpc = lib()
    r = torch.zeros(4, 32, device="cuda")
    v = torch.ones(32, device="cuda")
    with pytest.raises(ValueError):
        dpc.dp_norm_gate_fwd(r, r, v, v, v, kind="batch")
    with pytest.raises(ValueError):
        dpc.dp_norm_gate_fwd(r, r, v, v, v, b1=v)
    with pytest.raises(TypeError):
        dpc.dp_norm_gate_fwd(r, r, v, v, v, kind="layer")
    with pytest.raises(ValueError):
        dpc.dp_norm_gate_fwd(r[:3], r, v, v, v)
    with pytest.raises(TypeError):
        dpc.dp_norm_gate_fwd(r, r.half(), v, v, v)
    with pytest.raises(TypeError):
        dpc.dp_norm_gate_fwd(r, r, v.double(), v, v)
    with pytest.raises(ValueError):
        dpc.dp_norm_gate_fwd(r, r, v, v, v, gate=torch.zeros(3, device="cuda"))
    for eps in (0.0, -1.0, float("nan"), 1e-60):
        with pytest.raises(dpc.DPError) as err:
            dpc.dp_norm_gate_fwd(r, r, v, v, v, eps=eps)
        assert err.value.code == dpc.DP_ERR_SHAPE
    long = torch.zeros(1, 16385, device="cuda")
    with pytest.raises(dpc.DPError) as err:
        dpc.dp_norm_gate_fwd(long, long, long[0], long[0], long[0])
    assert err.value.code == dpc.DP_ERR_UNSUPPORTED
    st = torch.zeros(4, 4, device="cuda")
    with pytest.raises(dpc.DPError) as err:
        dpc.dp_norm_gate_grad(r, r, v, v, v, st, r, r, work=torch.empty(64, dtype=torch.uint8, device="cuda"))
    assert err.value.code == dpc.DP_ERR_SHAPE


@pytest.mark.parametrize("dtype", ROWS[1:], ids=IDS[1:])
@pytest.mark.parametrize("T,H,kind,gate", [(30003, 1003, "layer", "full"), (60001, 259, "rms", "token"), (14700, 2039, "layer", "token"),
                                           (30000, 1021, "rms", "full"), (20000, 1538, "layer", "none")])
def test_many_rows_of_odd_lengths(dtype, T, H, kind, gate):
    """Enough rows for the bulk copies of the words under them: rows at the start, the end and in between, and the
    column sums over all rows (in f64 torch on the same stats), with the bounds of the tests above."""
    dpc = lib()
    g = torch.Generator(device="cuda").manual_seed(T + H)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    layer = kind == "layer"
    wd = wtype(dtype)
    t = {n: (rn(T, H) * (3.0 if n == "f" else 1.0) + (0.5 if n == "f" else 0.0)).to(dtype) for n in ("r", "f", "dr2", "du")}
    t["gate"] = None if gate == "none" else (rn(*((T, H) if gate == "full" else (T,))) * 0.5 + 0.5).to(dtype)
    for n, c in (("a", 0.1), ("w1", 1.0), ("w2", 1.0), ("b1", 0.0), ("b2", 0.0)):
        t[n] = (rn(H) * 0.1 + c).to(wd) if layer or n[0] != "b" else None
    r2, u, st = dpc.dp_norm_gate_fwd(*(t[n] for n in ("r", "f", "a", "w1", "w2", "b1", "b2", "gate")), kind, EPS)
    got = dpc.dp_norm_gate_grad(r2, *(t[n] for n in ("f", "a", "w1", "w2")), st, t["dr2"], t["du"], t["b1"], t["b2"], t["gate"], kind)
    rows = np.unique(np.concatenate([np.arange(40), T - 1 - np.arange(40), np.random.default_rng(1).integers(0, T, 200)]))
    at = torch.from_numpy(rows).cuda()
    host = lambda x, whole: np.zeros(H) if x is None else f64(x if whole else x[at])  # noqa: E731
    d = {n: (None, host(t[n], n in ("a", "w1", "w2", "b1", "b2"))) for n in t if n != "gate"}
    d["gate"] = (None, np.ones(1) if gate == "none" else f64(t["gate"][at]))
    rr, ru, rst = forward(d, kind)
    a, un = 128 * SUM_UNIT[dtype], UNIT[dtype]
    big = lambda v: 1 + np.abs(v).max(1, keepdims=True)  # noqa: E731
    mag, mag2 = 1 + np.abs(d["f"][1]).max(1, keepdims=True) * rst[:, 1:2], 1 + np.abs(rr).max(1, keepdims=True) * rst[:, 3:4]
    within(r2[at], rr, un * np.abs(rr) + a * big(rr) * mag + TINY[dtype], "r2")
    within(u[at], ru, un * np.abs(ru) + a * big(ru) * mag * mag2 + TINY[dtype], "u")
    back, _, (s1, s2, n1, n2, p, dg) = backward(d, f64(r2[at]), f64(st[at]), kind, gate)
    top = lambda v: np.abs(v).max(1, keepdims=True)  # noqa: E731
    dr_mag = (top(d["dr2"][1]) + s2 * top(d["du"][1] * d["w2"][1]) * (1 + top(n2) ** 2)) * np.ones((1, H))
    within(got["dr"][at], back["dr"], un * np.abs(back["dr"]) + 2 * a * dr_mag + TINY[dtype], "dr")
    G = 1.0 if gate == "none" else np.abs(d["gate"][1]).reshape(len(rows), -1)
    df_mag = s1 * top(dr_mag * np.abs(d["a"][1] * d["w1"][1]) * G) * (1 + top(n1) ** 2)
    within(got["df"][at], back["df"], un * np.abs(back["df"]) + 4 * a * df_mag + TINY[dtype], "df")
    if gate != "none":
        dg_mag = dr_mag * np.abs(d["a"][1]) * (np.abs(p) + np.abs(d["b1"][1]) + np.abs(n1))
        dg_mag = dg_mag if gate == "full" else dg_mag.sum(1)
        within(got["dgate"][at], back["dgate"], un * np.abs(back["dgate"]) + 4 * a * dg_mag + TINY[dtype], "dgate")
    # column sums: dr as computed (unrounded dr differs from it by its rounding, in the bound)
    D = {n: None if x is None else x.double() for n, x in t.items()}
    s = st.double()
    N1, N2 = (D["f"] - s[:, :1]) * s[:, 1:2], (r2.double() - s[:, 2:3]) * s[:, 3:4]
    Gt = torch.ones(T, 1, device="cuda", dtype=torch.float64) if gate == "none" else D["gate"].reshape(T, -1)
    P = N1 * D["w1"] + (D["b1"] if layer else 0.0)
    dr, DP = got["dr"].double(), got["dr"].double() * D["a"] * Gt
    cols = {"da": dr * Gt * P, "dw1": DP * N1, "dw2": D["du"] * N2}
    if layer:
        cols.update(db1=DP, db2=D["du"])
    for n, c in cols.items():
        bound = (un if n in ("da", "dw1", "db1") else 0.0) * c.abs().sum(0)
        bound = bound + (4 * a + (T // 152 + 64) * SUM_UNIT[dtype]) * (c.abs() + dr.abs().mean() * 1e-3).sum(0)
        within(got[n], f64(c.sum(0)), f64(bound), n)
