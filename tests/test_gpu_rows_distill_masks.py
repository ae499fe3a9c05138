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
