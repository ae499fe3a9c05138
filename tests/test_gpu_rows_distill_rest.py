"""GPU: the training loss of students that are sure of a listed token: what the target gives to the rest stands against a share of any
smallness, in the loss and in both forms of the gradient."""
import numpy as np
import pytest
import torch

from oracle import rows as ref
from rows_util import LOWEST, TYPES, device_rows, exact_values
from test_gpu_rows_distill import grad_alone, loss

pytestmark = pytest.mark.gpu
GAPS = (20.0, 40.0, 44.0, 45.0, 60.0, 80.0, 86.0, 88.0, 120.0, 700.0, 1e6, 5e7)


def sure_students(M, V, kind, inv_temp, seed, offset=0.0):
    """Rows whose first listed entry lies GAPS[r] (behind the temperature) above everything outside the list; the target gives half of its
    mass to the list.  Labels: the listed one, another one of the list, one outside, none."""
    g = np.random.default_rng(seed)
    K = 4
    x = np.clip(g.normal(size=(M, V)) * 2.0, -8.0, 8.0)
    x[::3] = 0.0                                              # (every third row: all others equal)
    idx = np.stack([g.permutation(V)[:K] for _ in range(M)]).astype(np.int32)
    label = np.empty(M, dtype=np.int32)
    for r in range(M):
        top = x[r].max() + GAPS[r % len(GAPS)] / inv_temp
        x[r, idx[r, 0]] = top
        x[r, idx[r, 1]] = top - 3.0
        label[r] = (idx[r, 0], idx[r, 1], np.setdiff1d(np.arange(64), idx[r])[0], -1)[r // len(GAPS) % 4]
    t = device_rows((x + offset).astype(np.float32), kind)
    p = np.tile(np.array([0.3, 0.1, 0.06, 0.04]), (M, 1))
    val = (np.log(p) / inv_temp).astype(np.float32)
    return t, exact_values(t), val, idx, np.zeros(M, dtype=np.float32), label


def check(kind, z, val, idx, t_lse, label, dloss, inv_temp, w, kl, ce, grads):
    for r in range(z.shape[0]):
        a, b, g = ref.distill(z[r], val[r].astype(np.float64), idx[r], float(t_lse[r]), int(label[r]), inv_temp, w[0], w[1], float(dloss[r]))
        # a temperature that 32 bits round (two roundings: 2 * 2^-24 of the logits' distance), sums to 2e-6, one rounding
        far = (z[r].max() - z[r].min()) * max(inv_temp, 1.0)
        assert abs(kl[r] - a) <= 2.0 ** -23 * far + 2e-6 + 2.0 ** -23 * abs(a), (r, kl[r], a)
        assert abs(ce[r] - b) <= 2.0 ** -23 * far + 2e-6 + 2.0 ** -23 * abs(b), (r, ce[r], b)
        # Outside the list an entry's gradient is s - p_rest * its share of the rest, both to these shares of themselves: the exponent's
        # temperature (2^-23 of its distance from the rest's largest logit), its argument's rounding (2^-24 of up to that and 130 powers of
        # two), the exponential 2^-22, the sum 1e-6, factors held in 20 bits (two of them 2^-20).  Listed: s to the same, p to 1e-6; so the label's weight.
        outside = np.ones(z.shape[1], dtype=bool)
        outside[idx[r]] = False
        picked = ~outside
        if label[r] >= 0:
            picked[label[r]] = True
        rest = np.where(outside, z[r] * inv_temp, -np.inf)
        share = np.exp(rest - ref.lse(rest))
        s, s1 = (np.exp(z[r] * it - ref.lse(z[r] * it)) for it in (inv_temp, 1.0))
        spread = np.where(outside, rest.max() - rest, 0.0) * max(inv_temp, 1.0) / inv_temp
        rel = 2.0 ** -22 * spread + 130 * 2.0 ** -24 + 2.0 ** -22 + 1e-6 + 4 * 2.0 ** -20
        near = 2.0 ** -22 * np.minimum(far, 60.0) + rel       # (listed ones, and shares at temperature 1: what is further off has no mass)
        scale = abs(float(dloss[r])) * (w[0] * inv_temp + w[1])
        bound = torch.finfo(TYPES[kind]).eps / 2 * np.abs(g) + scale * (rel * share + near * (s + s1) + 1e-6 * picked + 1e-17)
        for grad in grads:
            got = exact_values(grad)[r]
            assert np.isfinite(got).all(), r
            assert (np.abs(got - g) <= bound).all(), (r, np.argmax(np.abs(got - g) - bound), got[idx[r]], g[idx[r]])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,inv_temp,offset", [(48, 1000, 1.0, 0.0), (48, 1000, 8.0, 0.0), (48, 1000, 0.5, 0.0), (48, 1003, 1.25, -1e4), (48, 60000, 1.0, 0.0),
                                                 (48, 60000, 1.25, 0.0), (12, 152064, 0.5, 0.0), (300, 777, 1.5, 0.0)])
@pytest.mark.parametrize("loss_scale", [1.0, 65536.0])
def test_a_student_sure_of_a_listed_token(kind, M, V, inv_temp, offset, loss_scale):
    w = (1.0, 0.25)
    t, z, val, idx, t_lse, label = sure_students(M, V, kind, inv_temp, V, offset)
    dloss = np.full(M, loss_scale, dtype=np.float32)
    fused, apart = torch.zeros_like(t), torch.zeros_like(t)
    kl, ce, stats = loss(t, val, idx, t_lse, label, inv_temp, w, dloss, fused)
    grad_alone(t, val, idx, t_lse, label, inv_temp, w, stats, dloss, apart)
    alone, _, _ = loss(t, val, idx, t_lse, label, inv_temp, w, want_stats=False)
    np.testing.assert_array_equal(kl, alone)
    check(kind, z, val, idx, t_lse, label, dloss, inv_temp, w, kl, ce, [fused, apart])


def test_the_loss_grows_with_the_gap():
    """One listed token at z, the others at 0, the target half on it: kl = log(1/2) - (0 + log 999 - z) / 2 (the student's log-sum-exp is z to
    e^-79), its gradient there 1 - 1/2."""
    gaps = np.array([86.0, 88.0, 90.0, 200.0], dtype=np.float32)
    x = np.zeros((4, 1000), dtype=np.float32)
    x[:, 7] = gaps
    t = device_rows(x, "f32")
    grad = torch.zeros_like(t)
    half = np.full((4, 1), np.log(0.5), dtype=np.float32)
    kl, _, _ = loss(t, half, np.full((4, 1), 7, dtype=np.int32), np.zeros(4, dtype=np.float32), None, 1.0, (1.0, 0.0), None, grad)
    np.testing.assert_allclose(kl, np.log(0.5) - (np.log(999) - gaps) / 2, rtol=1e-6)
    np.testing.assert_allclose(grad[:, 7].cpu().numpy(), 0.5, rtol=1e-6)
    np.testing.assert_allclose(grad[:, 8].cpu().numpy(), -0.5 / 999, rtol=1e-5)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_in_the_logits_place(kind):
    t, z, val, idx, t_lse, label = sure_students(48, 20001, kind, 1.25, 5)
    dloss = np.ones(48, dtype=np.float32)
    want = torch.zeros_like(t)
    _, _, stats = loss(t, val, idx, t_lse, label, 1.25, (1.0, 0.25), dloss, want)
    apart = torch.zeros_like(t)
    grad_alone(t, val, idx, t_lse, label, 1.25, (1.0, 0.25), stats, dloss, apart)
    one, two = t.clone(), t.clone()
    loss(one, val, idx, t_lse, label, 1.25, (1.0, 0.25), dloss, one)
    grad_alone(two, val, idx, t_lse, label, 1.25, (1.0, 0.25), stats, dloss, two)
    assert torch.equal(one, want) and torch.equal(two, apart)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("mask", ["infinity", "lowest", "far"])
@pytest.mark.parametrize("M,V", [(6, 40000), (200, 999)])
def test_a_student_that_masks_everything_outside_the_entries(kind, mask, M, V):
    """A target that masks the same: its p_rest is a rounding, and no loss.  One that gives the rest half of its mass: an infinite loss, as of
    a listed token that the student masks."""
    g = np.random.default_rng(V)
    K, w, inv_temp = 12, (1.0, 0.25), 1.25
    x = np.full((M, V), {"infinity": -np.inf, "lowest": LOWEST[kind], "far": -1e9}[mask])
    idx = np.stack([g.permutation(V)[:K] for _ in range(M)]).astype(np.int32)
    np.put_along_axis(x, idx.astype(np.int64), g.normal(size=(M, K)) * 2.0, axis=1)
    t = device_rows(x.astype(np.float32), kind)
    z = exact_values(t)
    val, label, dloss = (g.normal(size=(M, K)) * 2.0).astype(np.float32), idx[:, 3].copy(), np.ones(M, dtype=np.float32)
    t_lse = np.array([ref.lse(v * inv_temp) for v in val.astype(np.float64)], dtype=np.float32)
    for rest, lse in (("none", t_lse), ("half", t_lse + np.float32(np.log(2.0)))):
        fused, apart = torch.zeros_like(t), torch.zeros_like(t)
        kl, ce, stats = loss(t, val, idx, lse, label, inv_temp, w, dloss, fused)
        grad_alone(t, val, idx, lse, label, inv_temp, w, stats, dloss, apart)
        want = [ref.distill(z[r], val[r].astype(np.float64), idx[r], float(lse[r]), int(label[r]), inv_temp, *w) for r in range(M)]
        assert np.isposinf([a for a, _, _ in want]).all() == (rest == "half")
        # as for the formula's other rows: sums to 2e-6 and one rounding; a gradient's terms to 8e-6 of at most 1, and its rounding
        for r, (a, b, grad) in enumerate(want):
            assert kl[r] == a if np.isinf(a) else abs(kl[r] - a) <= 2e-6 + 2.0 ** -23 * abs(a), (rest, r, kl[r], a)
            assert abs(ce[r] - b) <= 2e-6 + 2.0 ** -23 * abs(b)
            for got in (fused, apart):
                got = exact_values(got)[r]
                assert (np.abs(got - grad) <= torch.finfo(TYPES[kind]).eps / 2 * np.abs(grad) + 2 * 8e-6 * (grad != 0)).all(), (rest, r)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_a_label_whose_cross_entropy_is_out_of_range_and_counts_for_nothing(kind):
    """Logits whose size a flat temperature brings back in range: the cross-entropy at temperature 1 has none, kl and its gradient are as ever."""
    M, V, inv_temp, w = 24, 1003, 0.1, (1.0, 0.0)
    t, z, val, idx, t_lse, label = sure_students(M, V, kind, inv_temp, 11)
    dloss = np.ones(M, dtype=np.float32)
    fused, apart = torch.zeros_like(t), torch.zeros_like(t)
    kl, ce, stats = loss(t, val, idx, t_lse, label, inv_temp, w, dloss, fused)
    grad_alone(t, val, idx, t_lse, label, inv_temp, w, stats, dloss, apart)
    far = (z.max(axis=1) > 2.0 ** 28 * np.log(2.0)) & (label >= 0)
    assert far.any() and not far.all()
    np.testing.assert_array_equal(np.isnan(ce), far)
    for r in np.flatnonzero(far):
        ce[r] = ref.distill(z[r], val[r].astype(np.float64), idx[r], float(t_lse[r]), int(label[r]), inv_temp, *w)[1]
    check(kind, z, val, idx, t_lse, label, dloss, inv_temp, w, kl, ce, [fused, apart])
