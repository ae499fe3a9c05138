"""GPU: the training loss of students whose masked tokens have the type's lowest value: they have no share of the soft-max, wherever they lie."""
import numpy as np
import pytest
import torch

from oracle import rows as ref
from rows_util import LOWEST, device_rows, exact_values
from test_gpu_rows_distill import check_rows, grad_alone, loss

pytestmark = pytest.mark.gpu


def masked_rows(M, V, kind, seed):
    """Rows whose allowed tokens are a stretch in front, one behind, a window of 40, or any tenth."""
    g = np.random.default_rng(seed)
    x = np.clip(g.normal(size=(M, V)) * 2.0, -8.0, 8.0)
    at = np.arange(V)
    for r in range(M):
        first = int(g.integers(0, V - 40))
        allowed = (at < V // 3, at >= V - V // 3, (at >= first) & (at < first + 40), g.random(V) < 0.1)[r % 4]
        x[r, ~allowed] = LOWEST[kind]
    t = device_rows(x.astype(np.float32), kind)
    return t, exact_values(t), g


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("M,V,inv_temp", [(4, 60000, 1.0), (4, 152064, 1.25), (160, 3001, 1.0), (160, 3001, 0.5)])
def test_masks_of_the_lowest_value(kind, tail, M, V, inv_temp):
    K, w = 16, (0.9, 0.3)
    t, z, g = masked_rows(M, V, kind, M + V)
    val, idx = np.zeros((M, K), dtype=np.float32), np.zeros((M, K), dtype=np.int32)
    t_lse, label = np.zeros(M, dtype=np.float32), np.zeros(M, dtype=np.int32)
    for r in range(M):
        teacher = np.where(z[r] > -100.0, z[r] + 0.5 * g.normal(size=V), -np.inf)
        val[r], idx[r], t_lse[r] = ref.top(teacher, K, inv_temp)
        label[r] = g.choice(np.flatnonzero(z[r] > -100.0))
    dloss = g.uniform(0.2, 2.0, M).astype(np.float32)
    fused, apart = torch.zeros_like(t), torch.zeros_like(t)
    lse = t_lse if tail else None
    kl, ce, stats = loss(t, val, idx, lse, label, inv_temp, w, dloss, fused)
    grad_alone(t, val, idx, lse, label, inv_temp, w, stats, dloss, apart)
    check_rows(kind, z, val, idx, lse, label, dloss, inv_temp, w, kl, ce, [fused, apart])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("inv_temp", [1.0, 0.5, 4.0])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_where_logits_get_too_large(kind, inv_temp, sign):
    """Losses up to a largest logit of 2^28 ln 2 behind the temperature (without it for the cross-entropy), NaN beyond."""
    V, K, edge = 3000, 8, 2.0 ** 28 * np.log(2.0)
    g = np.random.default_rng(1)
    tops = sign * edge * np.array([0.98, 1.02, 0.98 / inv_temp, 1.02 / inv_temp])
    x = tops[:, None] - np.abs(g.normal(size=(4, V))) * 1e4
    idx = np.stack([g.permutation(V)[:K] for _ in range(4)]).astype(np.int32)
    x[np.arange(4), idx[:, 0]] = tops
    t = device_rows(x.astype(np.float32), kind)
    z = exact_values(t)
    val, label = (g.normal(size=(4, K))).astype(np.float32), idx[:, 1].copy()
    grad = torch.zeros_like(t)
    kl, ce, _ = loss(t, val, idx, None, label, inv_temp, (1.0, 0.5), None, grad)
    for r in range(4):
        a, b, _ = ref.distill(z[r], val[r].astype(np.float64), idx[r], None, int(label[r]), inv_temp, 1.0, 0.5)
        top, far = np.abs(z[r].max()), z[r].max() - z[r].min()
        # a temperature that 32 bits round (2^-23 of the distance), sums to 2e-6, one rounding
        assert np.isnan(kl[r]) if top * inv_temp > edge else abs(kl[r] - a) <= 2.0 ** -23 * inv_temp * far + 2e-6 + 2.0 ** -23 * abs(a), (r, kl[r], a)
        assert np.isnan(ce[r]) if top > edge else abs(ce[r] - b) <= 2.0 ** -23 * far + 2e-6 + 2.0 ** -23 * abs(b), (r, ce[r], b)
        if top * inv_temp < edge and top < edge:
            assert torch.isfinite(grad[r]).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_listed_tokens_and_labels_that_are_masked(kind):
    """Losses of the size of the lowest value, infinite where 32 bits do not hold them; the other rows as ever, and no gradient but the target's."""
    M, V, K = 8, 4099, 6
    t, z, g = masked_rows(M, V, kind, 3)
    val, idx, label = (g.normal(size=(M, K))).astype(np.float32), np.zeros((M, K), dtype=np.int32), np.zeros(M, dtype=np.int32)
    for r in range(M):
        allowed, masked = np.flatnonzero(z[r] > -100.0), np.flatnonzero(z[r] < -100.0)
        idx[r] = g.permutation(allowed)[:K]
        idx[r, 2] = masked[r]
        label[r] = masked[r + 1] if r % 2 else allowed[0]
    for tail in (False, True):
        lse = np.array([ref.lse(v) + 0.7 for v in val.astype(np.float64)], dtype=np.float32) if tail else None
        fused, apart = torch.zeros_like(t), torch.zeros_like(t)
        kl, ce, stats = loss(t, val, idx, lse, label, 1.0, (1.0, 0.25), None, fused)
        grad_alone(t, val, idx, lse, label, 1.0, (1.0, 0.25), stats, None, apart)
        for r in range(M):
            a, b, want = ref.distill(z[r], val[r].astype(np.float64), idx[r], None if lse is None else float(lse[r]), int(label[r]), 1.0, 1.0, 0.25)
            assert a > 1e36 and kl[r] == pytest.approx(a, rel=1e-6)
            assert ce[r] == pytest.approx(b, rel=1e-6, abs=2e-6)
            for grad in (fused, apart):
                got = exact_values(grad)[r]
                assert (np.abs(got - want) <= torch.finfo(t.dtype).eps / 2 * np.abs(want) + 2 * 8e-6 * (want != 0)).all(), r
