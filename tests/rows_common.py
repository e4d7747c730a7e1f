"""Helpers for the expert-block tests: inputs of a row type, unit roundoffs, and elementwise bounds."""
import numpy as np
import torch

ROWS = [torch.float64, torch.float32, torch.bfloat16, torch.float16]
IDS = ["f64", "f32", "bf16", "f16"]
# unit roundoff (half the spacing at 1) of a row type, and of what its sums are held in
UNIT = {t: torch.finfo(t).eps / 2 for t in ROWS}
SUM_UNIT = {torch.float64: 2.0 ** -53, torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -24, torch.float16: 2.0 ** -24}
TINY = {torch.float64: 0.0, torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def wtype(dtype):
    return torch.float64 if dtype == torch.float64 else torch.float32


def rnd(seed, *shape, dtype=torch.float64, scale=1.0, shift=0.0):
    """(CUDA tensor of dtype, the values it holds as f64 numpy)."""
    a = np.random.default_rng(seed).normal(shift, scale, shape)
    t = torch.from_numpy(a).to(dtype)
    return t.cuda(), t.double().numpy()


def f64(t):
    return t.detach().double().cpu().numpy()


def within(got, ref, bound, what=""):
    """|got - ref| <= bound elementwise (arrays)."""
    got, ref = f64(got) if isinstance(got, torch.Tensor) else got, np.asarray(ref)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    over = np.abs(got - ref) - bound
    assert got.size == 0 or not np.any(~(over <= 0)), f"{what}: beyond its bound by {np.nanmax(over):.3e}"


def offset_view(t, elems=1):
    """The same values in a contiguous tensor whose first element lies `elems` past a 256-byte boundary."""
    buf = torch.empty(t.numel() + elems, dtype=t.dtype, device=t.device)
    buf[elems:] = t.reshape(-1)
    return buf[elems:].view(t.shape)
