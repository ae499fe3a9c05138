"""GPU: the training loss and its gradient where copies do not come: the calls return and report it, whatever number of pieces and rows
still wait for their place in the ring, and write nothing beside the rows."""
import pytest
import torch

from paper_2509_18824_b200 import binding as sd
from rows_util import TYPES
from test_gpu_rows_distill import check_rows, grad_alone, loss, problem

pytestmark = pytest.mark.gpu
W = (1.0, 0.1)
# a row per CTA, several short rows, several rows of more pieces than the ring holds (one, two and four CTAs a row)
SHAPES = [(2, 3000), (700, 3001), (900, 9000), (160, 60001), (160, 152064)]


@pytest.fixture
def withheld(monkeypatch):
    """Copies that do not come, inside `with`."""
    class Withheld:
        def __enter__(self):
            monkeypatch.setenv("SDV_TEST_WAIT_CYCLES", "100000")
            monkeypatch.setenv("SDV_TEST_WITHHOLD", "1")

        def __exit__(self, *_):
            monkeypatch.delenv("SDV_TEST_WITHHOLD")
            monkeypatch.delenv("SDV_TEST_WAIT_CYCLES")
    return Withheld()


def with_gaps(M, V, kind):
    """(a gradient whose rows lie 31 apart, all that is beside its rows as a function)"""
    ld = V + 31
    whole = torch.full((M * ld + 4096,), 5.0, dtype=TYPES[kind], device="cuda")
    return whole[:M * ld].as_strided((M, V), (ld, 1)), lambda: torch.cat([whole[:M * ld].view(M, ld)[:, V:].reshape(-1), whole[M * ld:]])


def check_few(kind, p, kl, ce, grads):
    t, z, val, idx, t_lse, label, dloss = p
    few = slice(0, 8)
    check_rows(kind, z[few], val[few], idx[few], t_lse[few], label[few], None if dloss is None else dloss[few], 1.0, W, kl, ce, grads)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", SHAPES)
def test_loss_and_gradient(kind, M, V, withheld):
    p = t, _, val, idx, t_lse, label, dloss = problem(M, V, 16, kind, 4, True, 1.0)
    grad, beside = with_gaps(M, V, kind)
    with withheld:
        loss(t, val, idx, t_lse, label, 1.0, W, dloss, grad, status=sd.SD_ERR_TIMEOUT)
    assert (beside() == 5.0).all()
    kl, ce, _ = loss(t, val, idx, t_lse, label, 1.0, W, dloss, grad)
    check_few(kind, p, kl, ce, [grad])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", SHAPES)
def test_the_loss_alone(kind, M, V, withheld):
    p = t, _, val, idx, t_lse, label, _ = problem(M, V, 16, kind, 4, True, 1.0)
    with withheld:
        loss(t, val, idx, t_lse, label, 1.0, W, status=sd.SD_ERR_TIMEOUT)
    kl, ce, _ = loss(t, val, idx, t_lse, label, 1.0, W)
    check_few(kind, p, kl, ce, [])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", SHAPES)
def test_the_gradient_alone(kind, M, V, withheld):
    p = t, _, val, idx, t_lse, label, dloss = problem(M, V, 16, kind, 4, True, 1.0)
    kl, ce, stats = loss(t, val, idx, t_lse, label, 1.0, W)
    grad, beside = with_gaps(M, V, kind)
    with withheld:
        grad_alone(t, val, idx, t_lse, label, 1.0, W, stats, dloss, grad, status=sd.SD_ERR_TIMEOUT)
    assert (beside() == 5.0).all()
    grad_alone(t, val, idx, t_lse, label, 1.0, W, stats, dloss, grad)
    check_few(kind, p, kl, ce, [grad])
