"""Cases of the expert-block operators: routing atoms to experts and back, the 8-bit integer product with
token and channel scales, and the norms around a block with its gate and residual scale.

A "token" is an atom's feature row (a descriptor of M1 x M2 = 1600 values, or a hidden row of 240), an
"expert" one of several nets that share the atoms.  `run` makes one pass: in plain torch operations in
32 bits, or (own) through the package's entry points.  `exact` is the same from the definitions in 64 bits.
"""
import math

import numpy as np
import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ES = {"f32": 4, "bf16": 2, "f16": 2}


def _lib():
    import paper_2107_02103_gb300 as dpc
    return dpc


def listed():
    return [
        # an MD step's smallest call: four atoms, hidden rows, two experts each; all latency
        dict(name="route_few", op="route", T=4, k=2, E=8, H=240, dtype="f32", drop=0.0),
        # descriptors of a water box (12,288 atoms), two of eight experts each
        dict(name="route_water", op="route", T=12288, k=2, E=8, H=1600, dtype="bf16", drop=0.0),
        # many experts, odd row length (no row but the first is aligned), a sixth of the pairs over capacity
        dict(name="route_odd", op="route", T=30011, k=3, E=61, H=1003, dtype="f16", drop=0.16),
        # training or forces: the gradient of the same two moves on f32 descriptors
        dict(name="route_grad", op="route_grad", T=16384, k=2, E=8, H=1600, dtype="f32", drop=0.02),
        # one atom through two experts' first layers: every weight of those two is read once
        dict(name="i8_single", op="i8", T=1, k=2, E=8, K=1600, N=2048, dtype="f32", act="tanh"),
        # a screening batch through the first fitting layer 1600 -> 240 of four centre types
        dict(name="i8_first_layer", op="i8", T=65536, k=1, E=4, K=1600, N=240, dtype="f32", act="tanh"),
        # wide layers, one net: the largest product
        dict(name="i8_wide", op="i8", T=32768, k=1, E=1, K=2048, N=4096, dtype="bf16", act=""),
        # ragged experts and odd lengths everywhere
        dict(name="i8_odd", op="i8", T=2503, k=2, E=13, K=1237, N=517, dtype="f16", act="tanh"),
        # one atom's hidden row
        dict(name="norm_single", op="norm", T=1, H=240, dtype="f32", kind="rms", gate="full"),
        # a large screening batch of descriptors
        dict(name="norm_batch", op="norm", T=65536, H=1600, dtype="bf16", kind="layer", gate="full"),
        # training: gradients of rows and of the shared weights
        dict(name="norm_grad", op="norm_grad", T=24576, H=2048, dtype="f32", kind="rms", gate="full"),
        # odd rows, one gate value per atom
        dict(name="norm_grad_odd", op="norm_grad", T=9973, H=1003, dtype="f16", kind="layer", gate="token"),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    def most(case):
        """Halves the tokens until a case is no dearer than the largest listed ones."""
        while case["T"] > 1:
            w = work(case)
            if w["bytes"] <= 1.1e9 and w["flops"] <= 5.4e11 and case["T"] * case.get("k", 1) * case.get("H", case.get("K", 1)) <= 1.1e8:
                break
            case["T"] //= 2
        return case

    op = rng.choice(["route", "route_grad", "i8", "i8", "norm", "norm_grad"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    T = _log(rng, 1, 65536)
    width = _log(rng, 64, 4096)
    if rng.random() < 0.5:
        width = -(-width // 16) * 16
    if op in ("route", "route_grad"):
        E = _log(rng, 2, 128)
        return most(dict(op=op, T=T, k=min(E, rng.randint(1, 4)), E=E, H=width, dtype=dtype, drop=rng.choice([0.0, 0.05, 0.3])))
    if op == "i8":
        E = rng.choice([1, 1, _log(rng, 2, 32)])
        return most(dict(op=op, T=T, k=min(E, rng.randint(1, 2)), E=E, K=width, N=_log(rng, 32, 4096), dtype=dtype, act=rng.choice(["", "tanh"])))
    return most(dict(op=op, T=T, H=width, dtype=dtype, kind=rng.choice(["rms", "layer"]), gate=rng.choice(["none", "token", "full"])))


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _experts(g, T, k, E, drop):
    """k distinct experts per token, the lower ones more popular; a dropped pair is -1."""
    logit = -0.5 * torch.log(1.0 + torch.arange(E, device="cuda", dtype=torch.float32))
    noise = -torch.log(-torch.log(torch.rand(T, E, generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))
    expert = torch.topk(logit + noise, k, dim=1).indices.to(torch.int32)
    if drop:
        expert = torch.where(torch.rand(T, k, generator=g, device="cuda") < drop, torch.full_like(expert, -1), expert)
    return expert.contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, dt = case["op"], DT[case["dtype"]]
    s = dict(case=case)
    T = case["T"]
    if op in ("route", "route_grad"):
        k, E, H = case["k"], case["E"], case["H"]
        s["expert"] = _experts(g, T, k, E, case["drop"])
        s["w"] = torch.softmax(_rand(g, T, k), 1).contiguous()
        s["z"] = _rand(g, T * k, H).to(dt)  # the experts' outputs, in sorted order
        if op == "route":
            s["x"] = _rand(g, T, H).to(dt)
        else:
            s["start"], s["src"], s["pos"] = _plan(s["expert"], E)
            s["dy"] = _rand(g, T, H).to(dt)
            s["dxs"] = _rand(g, T * k, H).to(dt)
    elif op == "i8":
        k, E, K, N = case["k"], case["E"], case["K"], case["N"]
        ld = -(-K // 16) * 16
        # rows of different size with a few large channels, as hidden features have
        x = _rand(g, T, K) * torch.exp(0.5 * _rand(g, T, 1))
        x *= torch.where(torch.rand(K, generator=g, device="cuda") < 0.01, 8.0, 1.0)
        s["x"] = x.to(dt)
        wq = torch.zeros(E, N, ld, dtype=torch.int8, device="cuda")
        wq[:, :, :K] = (32.0 * _rand(g, E, N, K)).round().clamp(-127, 127).to(torch.int8)
        s["wq"] = wq
        s["sw"] = (0.5 + torch.rand(E, N, generator=g, device="cuda")) / (48.0 * math.sqrt(K))
        s["bias"] = 0.1 * _rand(g, E, N)
        s["start"] = s["src"] = s["pos"] = None
        if E > 1:
            s["start"], s["src"], s["pos"] = _plan(_experts(g, T, k, E, 0.0), E)
    else:
        H = case["H"]
        s["f"] = (3.0 * _rand(g, T, H) + 0.5).to(dt)
        s["a"] = 0.1 + 0.02 * _rand(g, H)  # residual scale per channel
        s["w1"], s["w2"] = 1.0 + 0.1 * _rand(g, H), 1.0 + 0.1 * _rand(g, H)
        layer = case["kind"] == "layer"
        s["b1"], s["b2"] = (0.1 * _rand(g, H), 0.1 * _rand(g, H)) if layer else (None, None)
        s["gate"] = None
        if case["gate"] != "none":
            s["gate"] = torch.sigmoid(_rand(g, *((T, H) if case["gate"] == "full" else (T,)))).to(dt)
        r = _rand(g, T, H).to(dt)
        if op == "norm":
            s["r"] = r
        else:
            s["r2"] = r
            s["dr2"], s["du"] = _rand(g, T, H).to(dt), _rand(g, T, H).to(dt)
            m1, s1 = _stats(s["f"].float(), layer)
            m2, s2 = _stats(r.float(), layer)
            s["stats"] = torch.cat([m1, s1, m2, s2], 1).contiguous()
    return s


EPS = 1e-6


# ------------------------------------------------------------------ plain forms


def _plan(expert, E):
    n = expert.numel()
    flat = expert.reshape(-1)
    key = torch.where((flat >= 0) & (flat < E), flat, torch.full_like(flat, E))
    sorted_key, order = torch.sort(key, stable=True)
    start = torch.searchsorted(sorted_key, torch.arange(E + 1, device=flat.device, dtype=key.dtype))
    rows = torch.arange(n, device=flat.device)
    kept = rows < start[E]
    src = torch.where(kept, order, torch.full_like(order, -1)).to(torch.int32)
    pos = torch.empty_like(order)
    pos[order] = torch.where(kept, rows, torch.full_like(rows, -1))
    return start, src, pos.to(torch.int32).reshape(expert.shape)


def _gather(x, src, k):
    return torch.where((src >= 0)[:, None], x[src.clamp(min=0).long() // k], torch.zeros((), dtype=x.dtype, device=x.device))


def _combine(z, pos, w):
    rows = z[pos.clamp(min=0).long()].float()
    scale = (pos >= 0).float() if w is None else torch.where(pos >= 0, w, torch.zeros_like(w))
    return (rows * scale[:, :, None]).sum(1).to(z.dtype)


def _plain_route(s):
    start, src, pos = _plan(s["expert"], s["case"]["E"])
    xs = _gather(s["x"], src, s["case"]["k"])
    return {"start": start, "src": src, "pos": pos, "xs": xs, "y": _combine(s["z"], pos, s["w"])}


def _plain_route_grad(s):
    pos, src, k, z = s["pos"], s["src"], s["case"]["k"], s["z"]
    dy = s["dy"].float()
    pair = src.clamp(min=0).long()
    scale = torch.where(src >= 0, s["w"].reshape(-1)[pair], torch.zeros((), device=z.device))
    dz = (dy[pair // k] * scale[:, None]).to(z.dtype)
    dw = (z[pos.clamp(min=0).long()].float() * dy[:, None, :]).sum(2)
    return {"dz": dz, "dw": torch.where(pos >= 0, dw, torch.zeros_like(dw)), "dx": _combine(s["dxs"], pos, None)}


def _quant(x):
    x = x.float()
    amax = x.abs().amax(1, keepdim=True)
    fine = amax >= 2.0 ** -100
    most = torch.full_like(amax, 127.0)  # a tensor: torch multiplies by a scalar's rounded reciprocal instead
    r = torch.where(fine, most / amax, torch.zeros_like(amax))
    return torch.round(x * r), torch.where(fine, amax / most, torch.zeros_like(amax))


def _plain_i8(s):
    K = s["case"]["K"]
    q, sx = _quant(s["x"])
    wq = s["wq"][:, :, :K].float()
    if s["start"] is None:
        y = (q @ wq[0].t()) * sx * s["sw"][0] + s["bias"][0]
    else:
        start, pair = s["start"], s["src"].long()
        q, sx = q[pair // s["case"]["k"]], sx[pair // s["case"]["k"]]
        rows = torch.arange(q.shape[0], device=q.device)
        e = torch.searchsorted(start, rows, right=True) - 1
        at = rows - start[e]
        padded = torch.zeros(s["case"]["E"], int((start[1:] - start[:-1]).max()), K, device=q.device)
        padded[e, at] = q
        y = torch.bmm(padded, wq.transpose(1, 2))[e, at] * sx * s["sw"][e] + s["bias"][e]
    if s["case"]["act"] == "tanh":
        y = torch.tanh(y)
    return {"y": y.to(s["x"].dtype), "sx": sx.reshape(-1)}


def _stats(v, layer):
    m = v.mean(1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
    return m, torch.rsqrt((v - m).square().mean(1, keepdim=True) + EPS)


def _plain_norm(s):
    dt, layer = s["f"].dtype, s["case"]["kind"] == "layer"
    f = s["f"].float()
    m1, s1 = _stats(f, layer)
    p = (f - m1) * s1 * s["w1"]
    if layer:
        p = p + s["b1"]
    g = s["gate"]
    if g is not None:
        p = p * (g.float()[:, None] if g.dim() == 1 else g.float())
    r2 = s["r"].float() + s["a"] * p
    m2, s2 = _stats(r2, layer)
    u = (r2 - m2) * s2 * s["w2"]
    if layer:
        u = u + s["b2"]
    return {"r2": r2.to(dt), "u": u.to(dt), "stats": torch.cat([m1, s1, m2, s2], 1)}


def _plain_norm_grad(s):
    dt, layer = s["f"].dtype, s["case"]["kind"] == "layer"
    m1, s1, m2, s2 = s["stats"].split(1, 1)
    n1, n2 = (s["f"].float() - m1) * s1, (s["r2"].float() - m2) * s2
    du = s["du"].float()
    t = du * s["w2"]
    dr = s["dr2"].float() + s2 * (t - n2 * (t * n2).mean(1, keepdim=True) - (t.mean(1, keepdim=True) if layer else 0.0))
    p = n1 * s["w1"] + s["b1"] if layer else n1 * s["w1"]
    g = s["gate"]
    G = None if g is None else g.float()[:, None] if g.dim() == 1 else g.float()
    gp, ga = (p, s["a"]) if G is None else (G * p, G * s["a"])
    dp = dr * ga
    t1 = dp * s["w1"]
    df = s1 * (t1 - n1 * (t1 * n1).mean(1, keepdim=True) - (t1.mean(1, keepdim=True) if layer else 0.0))
    out = {"dr": dr.to(dt), "df": df.to(dt), "da": (dr * gp).sum(0), "dw1": (dp * n1).sum(0), "dw2": (du * n2).sum(0)}
    if layer:
        out["db1"], out["db2"] = dp.sum(0), du.sum(0)
    if g is not None:
        dg = dr * s["a"] * p
        out["dgate"] = (dg.sum(1) if g.dim() == 1 else dg).to(dt)
    return out


# ------------------------------------------------------------------ one pass


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"route": _plain_route, "route_grad": _plain_route_grad, "i8": _plain_i8, "norm": _plain_norm, "norm_grad": _plain_norm_grad}[op](s)
    dpc = _lib()
    if op == "route":
        start, src, pos = dpc.dp_route_plan(s["expert"], c["E"])
        xs = dpc.dp_route_gather(s["x"], src, pos)
        return {"start": start, "src": src, "pos": pos, "xs": xs, "y": dpc.dp_route_combine(s["z"], pos, s["w"])}
    if op == "route_grad":
        dz, dw = dpc.dp_route_combine_grad(s["z"], src=s["src"], pos=s["pos"], w=s["w"], dy=s["dy"])
        return {"dz": dz, "dw": dw, "dx": dpc.dp_route_combine(s["dxs"], s["pos"])}
    if op == "i8":
        xq, sx = dpc.dp_quant_rows_i8(s["x"], src=s["src"], pos=s["pos"])
        y = dpc.dp_linear_i8(xq, sx, s["wq"], s["sw"], bias=s["bias"], start=s["start"], act=c["act"] or None, dtype=s["x"].dtype)
        return {"y": y, "sx": sx}
    kw = dict(b1=s["b1"], b2=s["b2"], gate=s["gate"], kind=c["kind"])
    if op == "norm":
        r2, u, stats = dpc.dp_norm_gate_fwd(s["r"], s["f"], s["a"], s["w1"], s["w2"], eps=EPS, **kw)
        return {"r2": r2, "u": u, "stats": stats}
    d = dpc.dp_norm_gate_grad(s["r2"], s["f"], s["a"], s["w1"], s["w2"], s["stats"], s["dr2"], s["du"], **kw)
    return {k: v for k, v in d.items() if v is not None}


def work(case):
    """Bytes and operations of one pass: each input read once, each output written once."""
    T, es = case["T"], ES[case["dtype"]]
    if case["op"] in ("route", "route_grad"):
        n, k, H, row = T * case["k"], case["k"], case["H"], case["H"] * es
        if case["op"] == "route":  # experts, weights; plan out; x, z in; xs, y out
            return {"bytes": 4 * n + 4 * n + 8 * (case["E"] + 1) + 8 * n + 2 * T * row + 2 * n * row, "flops": 2 * n * H}
        return {"bytes": 8 * n + 8 * n + (n + T) * row + n * row + (n + T) * row, "flops": 5 * n * H}
    if case["op"] == "i8":
        n, E, K, N = T * case["k"], case["E"], case["K"], case["N"]
        used = min(E, n)
        return {"bytes": T * K * es + used * N * (K + 8) + n * N * es + 4 * n + (8 * n + 8 * (E + 1) if E > 1 else 0), "flops": 2 * n * K * N}
    H = case["H"]
    gate = {"none": 0, "token": T, "full": T * H}[case["gate"]] * es
    nvec = 5 if case["kind"] == "layer" else 3
    if case["op"] == "norm":
        return {"bytes": 4 * T * H * es + gate + 16 * T + 4 * nvec * H, "flops": 14 * T * H}
    return {"bytes": 6 * T * H * es + 2 * gate + 16 * T + 8 * nvec * H, "flops": 32 * T * H}


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    d = lambda name: None if s[name] is None else s[name].double()  # noqa: E731

    def sum64(z, pos, w):
        """y[t] = sum over the kept j of w[t][j] z[pos[t][j]]."""
        y = torch.zeros(pos.shape[0], z.shape[1], dtype=torch.float64, device=z.device)
        for j in range(pos.shape[1]):
            t = np.flatnonzero(pos[:, j] >= 0)
            p = torch.from_numpy(pos[t, j]).long().to(z.device)
            t = torch.from_numpy(t).to(z.device)
            y[t] += z[p] if w is None else w[t, j, None] * z[p]
        return y

    if op == "route":
        expert, k, E = s["expert"].reshape(-1).cpu().numpy(), case["k"], case["E"]
        pairs = np.concatenate([np.flatnonzero(expert == e) for e in range(E)])
        pos = np.full(expert.size, -1, np.int64)
        pos[pairs] = np.arange(pairs.size)
        xs = torch.zeros(expert.size, case["H"], dtype=torch.float64, device="cuda")
        xs[: pairs.size] = d("x")[torch.from_numpy(pairs // k).cuda()]
        return {"start": None, "src": None, "pos": None, "xs": xs, "y": sum64(d("z"), pos.reshape(-1, k), d("w"))}
    if op == "route_grad":
        pos, k = s["pos"].cpu().numpy(), case["k"]
        dy, z, w = d("dy"), d("z"), d("w")
        dz, dw = torch.zeros_like(z), torch.zeros_like(w)
        for j in range(k):
            t = np.flatnonzero(pos[:, j] >= 0)
            t, p = torch.from_numpy(t).cuda(), torch.from_numpy(pos[t, j]).long().cuda()
            dz[p] = w[t, j, None] * dy[t]
            dw[t, j] = torch.einsum("th,th->t", z[p], dy[t])
        return {"dz": dz, "dw": dw, "dx": sum64(d("dxs"), pos, None)}
    if op == "i8":
        # the quantiser's 32-bit steps belong to its definition; all else in 64 bits
        x = s["x"].float().cpu().numpy()
        amax = np.abs(x).max(1)
        with np.errstate(divide="ignore"):
            r = np.where(amax >= np.float32(2.0 ** -100), np.float32(127.0) / amax, np.float32(0.0))
        q = torch.from_numpy(np.rint(x * r[:, None])).cuda().double()
        sx32 = torch.from_numpy(np.where(r > 0, amax / np.float32(127.0), np.float32(0.0))).cuda()
        sx, wq, sw, b = sx32.double(), d("wq")[:, :, : case["K"]], d("sw"), d("bias")
        if s["start"] is None:
            y = (q @ wq[0].t()) * torch.outer(sx, sw[0]) + b[0]
        else:
            tok = s["src"].long() // case["k"]
            at = s["start"].tolist()
            y = torch.zeros(tok.numel(), case["N"], dtype=torch.float64, device="cuda")
            for e in range(case["E"]):
                t = tok[at[e]: at[e + 1]]
                y[at[e]: at[e + 1]] = (q[t] @ wq[e].t()) * torch.outer(sx[t], sw[e]) + b[e]
            sx = sx[tok]
        return {"y": torch.tanh(y) if case["act"] == "tanh" else y, "sx": sx}
    layer = case["kind"] == "layer"
    f, a, w1, w2, b1, b2, g = (d(n) for n in ("f", "a", "w1", "w2", "b1", "b2", "gate"))
    G = torch.ones_like(f) if g is None else g.reshape(g.shape[0], -1).expand_as(f)

    def normed(v):
        m = v.mean(1) if layer else torch.zeros_like(v[:, 0])
        var = ((v - m[:, None]) ** 2).mean(1)
        return m, 1.0 / torch.sqrt(var + EPS)

    if op == "norm":
        m1, s1 = normed(f)
        n1 = (f - m1[:, None]) * s1[:, None]
        r2 = d("r") + a * G * (n1 * w1 + (b1 if layer else 0.0))
        m2, s2 = normed(r2)
        u = (r2 - m2[:, None]) * s2[:, None] * w2 + (b2 if layer else 0.0)
        return {"r2": r2, "u": u, "stats": torch.stack([m1, s1, m2, s2], 1)}
    m1, s1, m2, s2 = (c[:, None] for c in d("stats").unbind(1))
    r2, dr2, du = d("r2"), d("dr2"), d("du")
    H = case["H"]
    n1, n2 = (f - m1) * s1, (r2 - m2) * s2

    def back(dn, n, sc):  # through v -> (v - m) sc
        sub = n * (dn * n).sum(1, keepdim=True) / H
        return sc * (dn - sub - (dn.sum(1, keepdim=True) / H if layer else 0.0))

    dr = dr2 + back(du * w2, n2, s2)
    p = n1 * w1 + (b1 if layer else 0.0)
    dp = dr * a * G
    out = {"dr": dr, "df": back(dp * w1, n1, s1), "da": (dr * G * p).sum(0), "dw1": (dp * n1).sum(0), "dw2": (du * n2).sum(0)}
    if layer:
        out["db1"], out["db2"] = dp.sum(0), du.sum(0)
    if g is not None:
        dg = dr * a * p
        out["dgate"] = dg.sum(1) if g.dim() == 1 else dg
    return out
