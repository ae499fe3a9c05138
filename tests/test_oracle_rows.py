"""The reference of the operators on rows of logits against definitions spelled out: brute force over prefixes, frequencies,
differences of the loss."""
import numpy as np
import pytest

from oracle import rows


def test_order_breaks_ties_by_index_and_leaves_masked_entries_out():
    x = np.array([1.0, -np.inf, 3.0, np.nan, 3.0, -0.0, 0.0])
    assert rows.in_order(x).tolist() == [2, 4, 0, 5, 6]
    v, i, l = rows.top(x, 8, 2.0)
    assert i.tolist() == [2, 4, 0, 5, 6, -1, -1, -1] and v[5] == -np.inf
    assert l == pytest.approx(np.log(2 * np.exp(6) + np.exp(2) + 2))


@pytest.mark.parametrize("seed", range(6))
def test_kept_entries_by_brute_force(seed):
    g = np.random.default_rng(seed)
    x = np.round(g.normal(size=40) * 3, 1)                        # (ties)
    it, k, p, mp = 0.7, 25, 0.8, 0.02
    order = sorted(range(40), key=lambda v: (-x[v], v))[:k]
    mass = {v: np.exp(x[v] * it) for v in order}
    total = sum(mass.values())
    n = next(n for n in range(1, k + 1) if sum(mass[v] for v in order[:n]) >= p * total * (1 - 1e-13))
    want = [v for v in order[:n] if mass[v] >= mp * mass[order[0]]]
    got, _ = rows.keep(x, it, k, p, mp)
    assert got.tolist() == want


def test_draws_have_the_filtered_frequencies():
    x = np.log(np.array([0.1, 0.2, 0.3, 0.4]))
    p = rows.probabilities(x, top_k=3)
    assert p == pytest.approx([0, 2 / 9, 3 / 9, 4 / 9])
    us = (np.arange(9000) + 0.5) / 9000
    got = np.bincount([rows.draw(p, u)[0] for u in us], minlength=4)
    assert got.tolist() == [0, 2000, 3000, 4000]
    assert rows.draw(np.zeros(4), 0.5)[0] == -1


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences(tail):
    g = np.random.default_rng(3)
    V = 12
    z = g.normal(size=V)
    idx = np.array([4, 7, -1, 4, 0])                              # no entry, and the same index twice
    val = g.normal(size=5)
    t_lse = float(np.log(np.exp(val[idx >= 0] * 1.3).sum() * 1.6)) if tail else None
    f = lambda z: (lambda kl, ce, _: 0.9 * kl + 0.2 * ce)(*rows.distill(z, val, idx, t_lse, 7, 1.3, 0.9, 0.2))
    _, _, grad = rows.distill(z, val, idx, t_lse, 7, 1.3, 0.9, 0.2)
    for v in range(V):
        d = np.zeros(V)
        d[v] = 1e-6
        assert grad[v] == pytest.approx((f(z + d) - f(z - d)) / 2e-6, abs=2e-8)


def test_divergence_of_equal_distributions_is_zero():
    z = np.random.default_rng(0).normal(size=30)
    o = rows.in_order(z)[:6]
    kl, ce, g = rows.distill(z, z[o], o, rows.lse(z), -1, 1.0, 1.0, 1.0)
    assert abs(kl) < 1e-14 and ce == 0 and np.abs(g).max() < 1e-15


def test_a_student_that_masks_the_rest():
    """Infinite where the target has mass there, no term where that is a rounding's; a share of any smallness by its logarithm."""
    z = np.array([1.0, 0.0, -np.inf, -np.inf])
    idx, val = np.array([0, 1]), np.log(np.array([0.25, 0.25]))
    kl, _, g = rows.distill(z, val, idx, 0.0, -1, 1.0, 1.0, 0.0)
    s = np.exp(z[:2]) / np.exp(z[:2]).sum()
    assert np.isposinf(kl) and g == pytest.approx([s[0] - 0.25, s[1] - 0.25, 0, 0])
    t_lse = np.float32(rows.lse(val))
    kl, _, g = rows.distill(z, val, idx, float(t_lse), -1, 1.0, 1.0, 0.0)
    assert kl == pytest.approx(np.log(0.5) - 0.5 * np.log(s).sum(), abs=1e-6) and g == pytest.approx([s[0] - 0.5, s[1] - 0.5, 0, 0], abs=1e-6)
    z = np.array([2000.0, 0.0, 0.0])
    kl, _, g = rows.distill(z, np.log(np.array([0.5])), np.array([0]), 0.0, -1, 1.0, 1.0, 0.0)
    assert kl == pytest.approx(np.log(0.5) + 0.5 * (2000 - np.log(2))) and g == pytest.approx([0.5, -0.25, -0.25])
