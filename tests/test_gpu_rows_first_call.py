"""GPU: the sampled tail's first call, which makes its arrays, on another stream than the current one."""
import pytest
import torch

from paper_2509_18824_b200 import workloads as wl
from paper_2509_18824_b200.step import VerifyStep

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fused", [True, False])
def test_arrays_of_the_first_call_are_not_filled_behind_it(fused):
    w = wl.make("c5", B=2, L=1, V=1024, Hd=128, prefix=70, T=8)
    u, half = torch.full((2, 8), 0.3, device="cuda"), torch.full((2,), 0.5, device="cuda")
    want = VerifyStep(w)
    want.tail_sampled(1.0, u, half, fused=fused)
    vs = VerifyStep(w)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda._sleep(50000000)                              # the current stream is busy for some 25 milliseconds
    vs.tail_sampled(1.0, u, half, stream=side, fused=fused)
    torch.cuda.synchronize()
    vs.check_status()
    assert (want.lse_rows != 0).all()
    for a, b in ((vs.lse_rows, want.lse_rows), (vs.group_stats, want.group_stats), (vs.n_acc, want.n_acc), (vs.out_tok, want.out_tok), (vs.path, want.path)):
        assert torch.equal(a, b)
