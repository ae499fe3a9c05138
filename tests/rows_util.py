"""Rows of logits for the tests of the operators on them: patterns, device copies at any alignment, comparison with the oracle."""
import numpy as np
import torch

from oracle import rows as ref
from paper_2509_18824_b200 import binding as sd

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LOWEST = {"f32": float(np.finfo(np.float32).min), "bf16": float(torch.finfo(torch.bfloat16).min)}
PATTERNS = ("bulk", "peaks", "flat", "equal", "rising", "falling", "masked", "one", "none", "lowest", "all_lowest", "nan", "huge")


def row(kind, V, g, lowest):
    """One row of V logits (float64 values that float32 holds)."""
    x = g.normal(size=V) * 2.0
    if kind == "peaks":
        at = g.permutation(V)[:min(V, 12)]
        x[at] += 9.0 + 3.0 * g.random(at.size)
    elif kind == "flat":
        x *= 1e-3
    elif kind == "equal":
        x[:] = 1.25
    elif kind == "rising":
        x = np.sort(x)
    elif kind == "falling":
        x = np.sort(x)[::-1]
    elif kind == "masked":
        x[g.random(V) < 0.7] = -np.inf
    elif kind == "one":
        keep = g.integers(V)
        x = np.where(np.arange(V) == keep, x, -np.inf)
    elif kind == "none":
        x[:] = -np.inf
    elif kind == "lowest":
        x[g.random(V) < 0.7] = lowest
    elif kind == "all_lowest":
        x[:] = lowest
    elif kind == "nan":
        x[g.random(V) < 0.1] = np.nan
        x[g.random(V) < 0.1] = -np.inf
    elif kind == "huge":
        x = x * 1e4
    return x


def device_rows(x, kind, ld=None):
    """x [M, V] (numpy) on the GPU in rows `ld` apart; the space between holds NaN."""
    M, V = x.shape
    ld = V if ld is None else ld
    whole = torch.full((M * ld,), float("nan"), dtype=TYPES[kind], device="cuda")
    view = whole[:M * ld].as_strided((M, V), (ld, 1))
    view.copy_(torch.from_numpy(np.ascontiguousarray(x)).to(TYPES[kind]))
    return view


def exact_values(t):
    return t.double().cpu().numpy()


def margin(x, inv_temp, top_k, top_p, min_p):
    """How far (in shares of the mass) the row is from a border that rounding could move."""
    if inv_temp > np.float32(1e30):
        return 1.0
    o, z = ref.keep(x, inv_temp, top_k)
    if o.size == 0:
        return 1.0
    m = np.exp(z[o] - z[o[0]])
    c = np.cumsum(m)
    d = 1.0
    if top_p < 1.0:
        d = min(d, float(np.abs(c / c[-1] - top_p).min()))
    if min_p > 0.0:
        near = np.abs(m - min(min_p, 1.0))
        d = min(d, float(near[m < 1.0].min()) if (m < 1.0).any() else 1.0)
    return d
