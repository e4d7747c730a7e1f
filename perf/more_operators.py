"""Cases of the operators that stand before and beside an expert block: choosing experts from a router's logits and
the gradient of their weights, embeddings of ids (atom types) with the gradient by sorted ids, and the product of
rows and weights in microscaled 4-bit floating point.

A "token" is an atom's row (a descriptor of M1 x M2 = 1600 values, or a hidden row of 240), an "expert" one of
several nets that share the atoms.  `run` makes one pass: in plain torch operations in 32 bits (64 for the order of
nearly equal scores), or (own) through the package's entry points.  `exact` is the same from the definitions in
64 bits.
"""
import math

import torch

own = False

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ES = {"f32": 4, "bf16": 2, "f16": 2}


def _lib():
    import paper_2107_02103_gb300 as dpc
    return dpc


def listed():
    return [
        # an MD step's smallest call: four atoms choose two of eight nets
        dict(name="topk_few", op="topk", T=4, E=8, k=2, G=1, keep=1, top=1, score="softmax", bias=False, renorm=True, dtype="f32"),
        # a screening batch over many nets in groups, balanced by a bias; 16-bit logits tie often
        dict(name="topk_batch", op="topk", T=65536, E=128, k=6, G=8, keep=4, top=2, score="sigmoid", bias=True, renorm=True, dtype="bf16"),
        # training: the gradient of renormalised weights, nearly all of it zeros
        dict(name="topk_grad", op="topk_grad", T=65536, E=128, k=6, score="sigmoid", renorm=True, dtype="f32"),
        # plain softmax weights, whose gradient reaches every logit; odd rows
        dict(name="topk_grad_odd", op="topk_grad", T=30011, E=61, k=3, score="softmax", renorm=False, dtype="f16"),
        # four atoms' hidden rows get their type's row
        dict(name="embed_few", op="embed", T=4, V=118, H=240, add=True, drop=0.0, dtype="f32"),
        # a batch of descriptors plus the embedding of their atoms' elements
        dict(name="embed_batch", op="embed", T=65536, V=118, H=1600, add=True, drop=0.0, dtype="bf16"),
        # training on an alloy: four types share all rows, each sum is over thousands of them
        dict(name="embed_grad_types", op="embed_grad", T=65536, V=4, H=1600, drop=0.0, dtype="f32"),
        # a large table of which most rows are met once or never, a few often; padding ids, odd rows
        dict(name="embed_grad_table", op="embed_grad", T=24571, V=30011, H=1003, drop=0.03, dtype="f16"),
        # one atom through two nets' first layers
        dict(name="mx4_single", op="mx4", T=1, k=2, E=8, K=1600, N=2048, dtype="f32", act="tanh"),
        # a screening batch through the first fitting layer 1600 -> 240 of four centre types
        dict(name="mx4_first_layer", op="mx4", T=65536, k=1, E=4, K=1600, N=240, dtype="f32", act="tanh"),
        # wide layers, one net: the largest product
        dict(name="mx4_wide", op="mx4", T=32768, k=1, E=1, K=2048, N=4096, dtype="bf16", act=""),
        # ragged experts and odd lengths everywhere
        dict(name="mx4_odd", op="mx4", T=2503, k=2, E=13, K=1237, N=517, dtype="f16", act="tanh"),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, v))


def draw(rng):
    def most(case):
        """Halves the tokens until a case is no dearer than the largest listed ones."""
        while case["T"] > 1:
            w = work(case)
            wide = case["T"] * case.get("k", 1) * (case["K"] if case["op"] == "mx4" else case["E"]) if "k" in case else case["T"] * case["H"]
            if w["bytes"] <= 6.5e8 and w["flops"] <= 5.5e11 and wide <= (5.1e7 if case["op"].startswith("topk") else 1.1e8):
                break
            case["T"] //= 2
        return case

    op = rng.choice(["topk", "topk_grad", "embed", "embed_grad", "mx4", "mx4"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    T = _log(rng, 1, 65536)
    if op in ("topk", "topk_grad"):
        E = _log(rng, 2, 1024)
        k = min(E, rng.randint(1, 8))
        # one renormalised weight is 1 whatever the logits: no gradient
        case = dict(op=op, T=T, E=E, k=k, score=rng.choice(["softmax", "sigmoid"]), renorm=k > 1 and rng.random() < 0.5, dtype=dtype)
        if op == "topk":
            G = rng.choice([g for g in (1, 1, 2, 3, 4, 8, 16) if E % g == 0])
            keep = rng.randint(-(-case["k"] * G // E), G)  # enough groups to choose from
            case.update(G=G, keep=keep, top=rng.randint(1, 2), bias=rng.random() < 0.5)
        return most(case)
    width = _log(rng, 64, 4096)
    if rng.random() < 0.5:
        width = -(-width // 16) * 16
    if op == "mx4":
        E = rng.choice([1, 1, _log(rng, 2, 32)])
        return most(dict(op=op, T=T, k=min(E, rng.randint(1, 2)), E=E, K=width, N=_log(rng, 32, 4096), dtype=dtype, act=rng.choice(["", "tanh"])))
    V = _log(rng, 2, 32768)
    case = dict(op=op, T=T, V=min(V, int(1e8) // width), H=width, drop=rng.choice([0.0, 0.05]), dtype=dtype)
    if op == "embed":
        case["add"] = rng.random() < 0.5
    return most(case)


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _gumbel(g, *shape):
    return -torch.log(-torch.log(torch.rand(*shape, generator=g, device="cuda").clamp(1e-9, 1 - 1e-7)))


def _experts(g, T, k, E):
    """k distinct experts per token, the lower ones more popular."""
    logit = -0.5 * torch.log(1.0 + torch.arange(E, device="cuda", dtype=torch.float32))
    return torch.topk(logit + _gumbel(g, T, E), k, dim=1).indices.to(torch.int32).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, dt, T = case["op"], DT[case["dtype"]], case["T"]
    s = dict(case=case)
    if op in ("topk", "topk_grad"):
        E, k = case["E"], case["k"]
        s["x"] = (1.5 * _rand(g, T, E) + 0.5 * _rand(g, E)).to(dt)
        s["bias"] = 0.05 * _rand(g, E) if case.get("bias") else None
        if op == "topk_grad":
            s["expert"] = torch.topk(s["x"].float() + 0.1 * _gumbel(g, T, E), k, dim=1).indices.to(torch.int32).contiguous()
            s["dw"] = _rand(g, T, k)
    elif op in ("embed", "embed_grad"):
        V, H = case["V"], case["H"]
        # ids as frequent as 1 / rank, in an order of their own
        rank = torch.rand(T, generator=g, device="cuda").double().mul(math.log(V + 1.0)).exp().floor().long().sub(1).clamp(0, V - 1)
        ids = torch.randperm(V, generator=g, device="cuda")[rank]
        if case["drop"]:
            ids = torch.where(torch.rand(T, generator=g, device="cuda") < case["drop"], -1, ids)
        s["ids"] = ids.to(torch.int32)
        if op == "embed":
            s["W"] = _rand(g, V, H).to(dt)
            s["add"] = _rand(g, T, H).to(dt) if case["add"] else None
        else:
            s["dy"] = _rand(g, T, H).to(dt)
    else:
        k, E, K, N = case["k"], case["E"], case["K"], case["N"]
        # rows of different size with a few large channels, as hidden features have
        x = _rand(g, T, K) * torch.exp(0.5 * _rand(g, T, 1))
        x *= torch.where(torch.rand(K, generator=g, device="cuda") < 0.01, 8.0, 1.0)
        s["x"] = x.to(dt)
        # the weights' codes and scales, a row a channel: two codes a byte, the lower four bits first
        q, e = _quant((_rand(g, E * N, K) * (0.5 + torch.rand(E * N, 1, generator=g, device="cuda")) / math.sqrt(K)))
        code = torch.searchsorted(_grid(), q.abs().contiguous()) + 8 * (q < 0)
        s["wq"] = (code[:, 0::2] + 16 * code[:, 1::2]).to(torch.uint8).view(E, N, -1)
        sw = torch.zeros(E * N, -(-K // 256) * 8, dtype=torch.uint8, device="cuda")
        sw[:, : e.shape[1]] = (e + 127).to(torch.uint8)
        s["sw"] = sw.view(E, N, -1)
        s["bias"] = 0.1 * _rand(g, E, N)
        s["start"] = s["src"] = s["pos"] = None
        if E > 1:
            s["start"], s["src"], s["pos"] = _plan(_experts(g, T, k, E), E)
    return s


SCALE = 1.75  # of the chosen weights, and of embeddings


# ------------------------------------------------------------------ plain forms


def _order(v):
    """The indices of v's columns from the largest value on, equal ones by index."""
    return torch.sort(v, dim=1, descending=True, stable=True).indices


def _plain_topk(s):
    c = s["case"]
    x = s["x"].double()  # the order of scores next to each other
    score = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.exp(x - x.amax(1, keepdim=True))
    if c["score"] == "softmax":
        score = score / score.sum(1, keepdim=True)
    chosen_by = score if s["bias"] is None else score + s["bias"].double()
    order_by = x if s["bias"] is None else chosen_by
    if c["keep"] < c["G"]:
        per = c["E"] // c["G"]
        group = torch.topk(chosen_by.view(-1, c["G"], per), min(c["top"], per), dim=2).values.sum(2)
        kept = torch.zeros_like(group, dtype=torch.bool).scatter_(1, _order(group)[:, : c["keep"]], True)
        order_by = torch.where(kept.repeat_interleave(per, 1), order_by, -math.inf)
    expert = _order(order_by)[:, : c["k"]]
    w = score.float().gather(1, expert)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return {"expert": expert.to(torch.int32), "w": w * SCALE}


def _plain_topk_grad(s):
    c, e, dw = s["case"], s["expert"].long(), s["dw"] * SCALE
    x = s["x"].float()
    score = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.exp(x - x.amax(1, keepdim=True))
    if c["score"] == "softmax":
        score = score / score.sum(1, keepdim=True)
    at = score.gather(1, e)
    if c["renorm"]:
        n = at / at.sum(1, keepdim=True)
        dw = (dw - (dw * n).sum(1, keepdim=True)) / at.sum(1, keepdim=True)
    ds = torch.zeros_like(x).scatter_add_(1, e, dw)
    if c["score"] == "sigmoid":
        dx = ds * score * (1.0 - score)
    else:
        dx = score * (ds - (ds * score).sum(1, keepdim=True))
    return {"dx": dx.to(s["x"].dtype)}


def _plain_embed(s):
    ids = s["ids"].long()
    y = torch.where((ids >= 0)[:, None], s["W"][ids.clamp(min=0)].float() * SCALE, 0.0)
    if s["add"] is not None:
        y = s["add"].float() + y
    return {"y": y.to(s["W"].dtype)}


def _by_id(ids, V):
    key = torch.where((ids >= 0) & (ids < V), ids, V)
    sorted_key, order = torch.sort(key, stable=True)
    start = torch.searchsorted(sorted_key, torch.arange(V + 1, device=ids.device, dtype=key.dtype))
    return start, torch.where(sorted_key < V, order, -1).to(torch.int32)


def _plain_embed_grad(s):
    V, ids = s["case"]["V"], s["ids"]
    start, src = _by_id(ids, V)
    dW = torch.zeros(V + 1, s["dy"].shape[1], device=ids.device)
    dW.index_add_(0, torch.where(ids >= 0, ids, V).long(), s["dy"].float())
    return {"start": start, "src": src, "dW": dW[:V] * SCALE}


def _plan(expert, E):
    start, src = _by_id(expert.reshape(-1), E)
    pos = torch.empty_like(src)
    pos[src.long()] = torch.arange(src.numel(), device=src.device, dtype=torch.int32)  # no pair is dropped here
    return start, src, pos.reshape(expert.shape)


def _grid():
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")


def _quant(x):
    """x as 4-bit values and an exponent for 32 neighbours, both in columns up to a multiple of 64."""
    x = torch.nn.functional.pad(x.float(), (0, -x.shape[1] % 64)).view(x.shape[0], -1, 32)
    e = (torch.frexp(x.abs().amax(2, keepdim=True)).exponent - 3).clamp(min=-127)  # floor(log2) - 2
    v = x * ((127 - e) << 23).view(torch.float32)
    a = v.abs().clamp(max=6.0)
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    return (torch.copysign(torch.round(a / step) * step, v)).flatten(1), e.squeeze(2)


def _pow2(e):
    return torch.exp2(e.float()).repeat_interleave(32, 1)


def _plain_mx4(s):
    K, E, N = s["case"]["K"], s["case"]["E"], s["case"]["N"]
    q, e = _quant(s["x"])
    x = q * _pow2(e)
    code = torch.stack([s["wq"] & 15, s["wq"] >> 4], 3).flatten(2).long()
    w = torch.cat([_grid(), -_grid()])[code]
    w = (w.view(E * N, -1) * _pow2(s["sw"].view(E * N, -1)[:, : w.shape[2] // 32].int() - 127)).view(E, N, -1)
    if s["start"] is None:
        y = x @ w[0].t() + s["bias"][0]
    else:
        start, pair = s["start"], s["src"].long()
        x = x[pair // s["case"]["k"]]
        rows = torch.arange(x.shape[0], device=x.device)
        of = torch.searchsorted(start, rows, right=True) - 1
        at = rows - start[of]
        padded = torch.zeros(E, int((start[1:] - start[:-1]).max()), x.shape[1], device=x.device)
        padded[of, at] = x
        y = torch.bmm(padded, w.transpose(1, 2))[of, at] + s["bias"][of]
    if s["case"]["act"] == "tanh":
        y = torch.tanh(y)
    return {"y": y.to(s["x"].dtype)}


# ------------------------------------------------------------------ one pass


def run(s):
    c = s["case"]
    op = c["op"]
    if not own:
        return {"topk": _plain_topk, "topk_grad": _plain_topk_grad, "embed": _plain_embed, "embed_grad": _plain_embed_grad, "mx4": _plain_mx4}[op](s)
    dpc = _lib()
    if op == "topk":
        expert, w = dpc.dp_route_topk(s["x"], c["k"], bias=s["bias"], score=c["score"], ngroup=c["G"], keep_groups=c["keep"], group_top=c["top"], renorm=c["renorm"], scale=SCALE)
        return {"expert": expert, "w": w}
    if op == "topk_grad":
        return {"dx": dpc.dp_route_topk_grad(s["x"], s["expert"], s["dw"], score=c["score"], renorm=c["renorm"], scale=SCALE)}
    if op == "embed":
        return {"y": dpc.dp_embed_fwd(s["W"], s["ids"], scale=SCALE, add=s["add"])}
    if op == "embed_grad":
        start, src = dpc.dp_embed_plan(s["ids"], c["V"])
        return {"start": start, "src": src, "dW": dpc.dp_embed_grad(s["dy"], s["ids"], start, src, scale=SCALE)}
    xq, sx = dpc.dp_quant_rows_mx4(s["x"], src=s["src"], pos=s["pos"])
    return {"y": dpc.dp_linear_mx4(xq, sx, s["wq"], s["sw"], bias=s["bias"], start=s["start"], act=c["act"] or None, dtype=s["x"].dtype)}


def work(case):
    """Bytes and operations of one pass: each input read once, each output written once."""
    T, es, op = case["T"], ES[case["dtype"]], case["op"]
    if op == "topk":
        E, k = case["E"], case["k"]
        return {"bytes": T * E * es + (4 * E if case["bias"] else 0) + 8 * T * k, "flops": 8 * T * E}
    if op == "topk_grad":  # all logits only where every one has a gradient, else the chosen ones
        E, k = case["E"], case["k"]
        all_of = case["score"] == "softmax" and not case["renorm"]
        return {"bytes": T * E * es + (T * E if all_of else T * k) * es + 8 * T * k, "flops": (8 * T * E if all_of else 12 * T * k)}
    if op == "embed":
        H, V = case["H"], case["V"]
        return {"bytes": 4 * T + min(T, V) * H * es + (2 if case["add"] else 1) * T * H * es, "flops": 2 * T * H}
    if op == "embed_grad":
        H, V = case["H"], case["V"]
        return {"bytes": 8 * T + 8 * (V + 1) + T * H * es + 4 * V * H, "flops": T * H}
    n, E, K, N = T * case["k"], case["E"], case["K"], case["N"]
    return {"bytes": T * K * es + min(E, n) * N * (K // 2 + K // 32 + 4) + n * N * es + (8 * n + 8 * (E + 1) if E > 1 else 0), "flops": 2 * n * K * N}


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)

    def ranks(v):
        """For each value of a row, how many come before it: larger ones, and equal ones of a lower index."""
        n = v.shape[1]
        at = torch.arange(n, device=v.device)
        out = torch.empty(v.shape, dtype=torch.int64, device=v.device)
        step = max(1, int(6e7) // (n * n))
        for t in range(0, v.shape[0], step):
            a, b = v[t: t + step, :, None], v[t: t + step, None, :]
            out[t: t + step] = ((b > a) | ((b == a) & (at[None, :] < at[:, None]))).sum(2)
        return out

    def topk():
        x, E, k = s["x"].double(), case["E"], case["k"]
        if case["score"] == "sigmoid":
            score = 1.0 / (1.0 + torch.exp(-x))
        else:
            score = torch.exp(x - torch.logsumexp(x, 1, keepdim=True))
        c = score if s["bias"] is None else score + s["bias"].double()
        by = x if s["bias"] is None else c
        if case["keep"] < case["G"]:
            per = E // case["G"]
            parts = c.view(-1, case["G"], per).sort(2).values[:, :, -case["top"]:]
            out = ranks(parts.sum(2)) >= case["keep"]
            by = by.masked_fill(out[:, :, None].expand(-1, -1, per).reshape(by.shape), -math.inf)
        rank = ranks(by)
        w = torch.stack([(score * (rank == j)).sum(1) for j in range(k)], 1)
        if case["renorm"]:
            w = w / w.sum(1, keepdim=True)
        return {"expert": None, "w": SCALE * w}

    def topk_grad():
        x, e, dw = s["x"].double(), s["expert"].long(), s["dw"].double() * SCALE
        T, E = x.shape
        # d log(score_e) / dx_f = [e = f] (1 - score) for a sigmoid, [e = f] - score_f for a softmax
        score = 1.0 / (1.0 + torch.exp(-x)) if case["score"] == "sigmoid" else torch.exp(x - torch.logsumexp(x, 1, keepdim=True))
        at = torch.stack([score[torch.arange(T, device="cuda"), e[:, j]] for j in range(case["k"])], 1)
        w = at / at.sum(1, keepdim=True) if case["renorm"] else at
        coef = w * dw  # of d log(score) at each choice
        if case["renorm"]:
            coef = coef - w * coef.sum(1, keepdim=True)
        dx = torch.zeros_like(x)
        rows = torch.arange(T, device="cuda")
        for j in range(case["k"]):
            own_part = coef[:, j] * (1.0 - at[:, j]) if case["score"] == "sigmoid" else coef[:, j]
            dx[rows, e[:, j]] += own_part
        if case["score"] == "softmax" and not case["renorm"]:
            dx -= score * coef.sum(1, keepdim=True)
        return {"dx": dx}

    def mx4():
        def values(x):  # each 4-bit value from the places where two of them are equally near
            n, K = x.shape
            x = x.float().double()
            b = torch.zeros(n, -(-K // 32) * 32, dtype=torch.float64, device="cuda")
            b[:, :K] = x
            b = b.view(n, -1, 32)
            big = b.abs().amax(2, keepdim=True)
            up = torch.floor(torch.log2(big.clamp(min=2.0 ** -125)))
            up = torch.where(torch.exp2(up) > big, up - 1, up)
            unit = torch.exp2(torch.where(torch.exp2(up + 1) <= big, up + 1, up).clamp(min=-125.0) - 2)
            a = b.abs() / unit
            q = 0.5 * (a > 0.25) + 0.5 * (a >= 0.75) + 0.5 * (a > 1.25) + 0.5 * (a >= 1.75) + 1.0 * (a > 2.5) + 1.0 * (a >= 3.5) + 2.0 * (a > 5.0)
            return (torch.sign(b) * q * unit).flatten(1)

        E, N, K = case["E"], case["N"], case["K"]
        x = values(s["x"])
        Kp = x.shape[1]
        code = torch.zeros(E, N, 2 * s["wq"].shape[2], dtype=torch.int64, device="cuda")
        code[:, :, 0::2], code[:, :, 1::2] = s["wq"].long() % 16, s["wq"].long() // 16
        code = code[:, :, :Kp]
        mag, sign = code % 8, 1.0 - 2.0 * (code >= 8)
        w = sign * torch.where(mag < 2, mag * 0.5, torch.exp2((mag // 2 - 1).double()) * (1.0 + 0.5 * (mag % 2)))
        w = (w.view(E, N, -1, 32) * torch.exp2(s["sw"][:, :, : Kp // 32].double() - 127.0)[..., None]).flatten(2)
        b = s["bias"].double()
        if s["start"] is None:
            y = x @ w[0].t() + b[0]
        else:
            tok, at = s["src"].long() // case["k"], s["start"].tolist()
            y = torch.zeros(tok.numel(), N, dtype=torch.float64, device="cuda")
            for e in range(E):
                y[at[e]: at[e + 1]] = x[tok[at[e]: at[e + 1]]] @ w[e].t() + b[e]
        return {"y": torch.tanh(y) if case["act"] == "tanh" else y}

    op = case["op"]
    if op == "topk":
        return topk()
    if op == "topk_grad":
        return topk_grad()
    if op == "mx4":
        return mx4()
    ids = s["ids"].long()
    met = ids >= 0
    if op == "embed":
        y = torch.zeros(case["T"], case["H"], dtype=torch.float64, device="cuda") if s["add"] is None else s["add"].double()
        y[met] += SCALE * s["W"].double()[ids[met]]
        return {"y": y}
    dW = torch.zeros(case["V"], case["H"], dtype=torch.float64, device="cuda")
    dW.scatter_add_(0, ids[met][:, None].expand(-1, case["H"]), SCALE * s["dy"].double()[met])
    return {"start": None, "src": None, "dW": dW}
