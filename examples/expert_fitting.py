"""A mixture-of-experts block on Deep Potential descriptors, with the library's expert-block calls.

Each atom's descriptor row goes to `topk` of several nets that all atom types share, and comes back as their
weighted sum, normed, gated and scaled into the residual stream:

    u    = descriptor rows                                     [nloc][H]
    y_i  = sum_j w_ij net_{e_ij}(u_i)                          route, nets, combine
    r2   = r + a gate norm(y);   u2 = norm(r2)                 one pass
    E    = sum_i <u2_i, v>

Two ways through the nets: in f64 or f32 with dp_fitting_* (values, and the gradient dE/du that the forces need), and
in 8-bit integers (values only: ranking many candidate structures).

    python examples/expert_fitting.py          # needs a GPU and the built library
"""
from __future__ import annotations

import os
import sys
from dataclasses import dataclass

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2107_02103_gb300 as dpc  # noqa: E402


@dataclass
class ExpertBlock:
    """Nets of one tanh layer, H -> hidden -> H, as dp_fitting_* parameters, and the weights around them."""
    params: torch.Tensor  # [nexp][P]
    widths: tuple
    a: torch.Tensor  # residual scale [H]
    w1: torch.Tensor  # norm weights [H]
    w2: torch.Tensor
    v: torch.Tensor  # energy weights [H]
    kind: str = "rms"
    i8: tuple | None = None

    @classmethod
    def random(cls, seed, nexp, H, hidden, dtype=torch.float64, device="cuda"):
        g = torch.Generator(device="cpu").manual_seed(seed)
        rn = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
        nets = [torch.cat([rn(H * hidden) / H ** 0.5, 0.1 * rn(hidden), rn(hidden * H) / hidden ** 0.5, 0.1 * rn(H)])
                for _ in range(nexp)]
        vec = [0.5 + 0.05 * rn(H), 1.0 + 0.1 * rn(H), 1.0 + 0.1 * rn(H), rn(H) / H ** 0.5]
        to = lambda t: t.to(dtype).to(device)  # noqa: E731
        return cls(to(torch.stack(nets)), (H, hidden, H), *(to(t) for t in vec))

    def forward(self, u, expert, weight, gate=None):
        """E, and what backward needs."""
        start, src, pos = dpc.dp_route_plan(expert, self.params.shape[0])
        # the nets take their rows by sorted ranges that the host knows; rows past the kept ones go to none
        ends = start.tolist()
        xs = dpc.dp_route_gather(u, src, pos)
        z = torch.zeros_like(xs)
        kept = ends[-1]
        z[:kept], act = dpc.dp_fitting_fwd(self.params, self.widths, ends, xs[:kept])
        y = dpc.dp_route_combine(z, pos, weight)
        r2, u2, stats = dpc.dp_norm_gate_fwd(u, y, self.a, self.w1, self.w2, gate=gate, kind=self.kind)
        return (u2 @ self.v).sum(), (ends, src, pos, weight, gate, z, act, y, r2, stats)

    def backward(self, saved):
        """dE/du, dE/dweight (the router's), and a dict of dE/da, dw1, dw2 and dgate."""
        ends, src, pos, weight, gate, z, act, y, r2, stats = saved
        du2 = self.v.expand_as(r2).contiguous()
        g = dpc.dp_norm_gate_grad(r2, y, self.a, self.w1, self.w2, stats, torch.zeros_like(r2), du2, gate=gate,
                                  kind=self.kind)
        dz, dweight = dpc.dp_route_combine_grad(z, src, pos, weight, g["df"])
        dxs = torch.zeros_like(dz)
        dxs[:ends[-1]] = dpc.dp_fitting_grad(self.params, self.widths, ends, act, dz[:ends[-1]])
        du = dpc.dp_route_combine(dxs, pos) + g["dr"]  # the gather's gradient, and the residual stream's
        return du, dweight, g

    def quantise(self):
        """The nets' weights as 8-bit rows, once."""
        H, hidden, _ = self.widths
        n = self.params.shape[0]
        W1, b1, W2, b2 = torch.split(self.params, [H * hidden, hidden, hidden * H, H], dim=1)
        layers = []
        for W, b, k, m in ((W1, b1, H, hidden), (W2, b2, hidden, H)):
            q, s = dpc.dp_quant_rows_i8(W.reshape(n, k, m).transpose(1, 2).reshape(n * m, k).contiguous())
            layers.append((q.view(n, m, -1), s.view(n, m), b.float().contiguous()))
        self.i8 = tuple(layers)
        return self

    def screen(self, u, expert, weight, gate=None):
        """Atomic energies <u2_i, v> with the nets in 8-bit integers; nothing waits for the host."""
        (q1, s1, b1), (q2, s2, b2) = self.i8
        start, src, pos = dpc.dp_route_plan(expert, self.params.shape[0])
        xq, sx = dpc.dp_quant_rows_i8(u, src, pos)
        h = dpc.dp_linear_i8(xq, sx, q1, s1, b1, start, act="tanh", dtype=u.dtype)
        hq, sh = dpc.dp_quant_rows_i8(h)
        z = dpc.dp_linear_i8(hq, sh, q2, s2, b2, start, dtype=u.dtype)
        y = dpc.dp_route_combine(z, pos, weight)
        _, u2, _ = dpc.dp_norm_gate_fwd(u, y, self.a, self.w1, self.w2, gate=gate, kind=self.kind)
        return u2 @ self.v


def route(logits, topk):
    """Experts and weights of each atom from the router's logits [nloc][nexp]."""
    top = torch.topk(logits, topk, dim=1)
    return top.indices.to(torch.int32), torch.softmax(top.values, dim=1)


def descriptors(dtype=torch.float64):
    """D [nloc][M1 M2] of a small synthetic copper box through the compressed model."""
    import workloads as W
    w = W.make("tiny")
    info = dpc.dp_table_info_make(w.s_min, w.s_max, w.stride0, w.stride1, w.ext)
    model = dpc.Model.compress(torch.from_numpy(w.params).cuda(), w.widths, info)
    dev = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
    T = dpc.dp_tabulate_fusion_fwd(model.table, info, dev(w.s), dev(w.Rt), dev(w.nvalid), dev(w.atype), w.sel)
    D = dpc.dp_descriptor_contract(T, w.M2).flatten(1)
    return (D / D.abs().mean()).to(dtype).contiguous()


def main():
    u = descriptors()
    block = ExpertBlock.random(1, 8, u.shape[1], 96)
    logits = torch.randn(u.shape[0], 8, dtype=torch.float64, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    expert, weight = route(logits, 2)
    E, saved = block.forward(u, expert, weight)
    du, dweight, _ = block.backward(saved)
    print(f"{u.shape[0]} atoms, descriptors of {u.shape[1]}: E = {float(E):.9f}, |dE/du| = {float(du.norm()):.6f}, "
          f"|dE/dweight| = {float(dweight.norm()):.6f}")
    low = ExpertBlock(*(t.float() if isinstance(t, torch.Tensor) else t for t in
                        (block.params, block.widths, block.a, block.w1, block.w2, block.v))).quantise()
    e8 = low.screen(u.float(), expert, weight.float())
    print(f"in 8-bit integers: E = {float(e8.double().sum()):.6f}")


if __name__ == "__main__":
    main()
