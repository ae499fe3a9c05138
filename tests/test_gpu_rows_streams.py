"""GPU: sampling parameters and a step's own buffers where the calls run on another stream than the current one, which is busy."""
import numpy as np
import pytest
import torch

from paper_2509_18824_b200 import binding as sd
from test_gpu_rows_sampling import batch, parameters

pytestmark = pytest.mark.gpu
BUSY = 100_000_000                                            # cycles of the current stream: some 50 ms


def outputs(M, V):
    return torch.zeros((M, V), device="cuda"), torch.zeros(M, device="cuda"), torch.zeros(M, dtype=torch.int32, device="cuda"), sd.new_status()


@pytest.mark.parametrize("as_argument", [True, False])
def test_parameters_that_are_converted_on_a_busy_stream(as_argument):
    """Tensors of other types on the GPU, handed to the call on another stream at once, and dropped behind it."""
    M, V = 12, 5000
    t, _ = batch(M, V, "f32", 3)
    it, k, p, mp = parameters(M, V, 3, "kpm")
    want = outputs(M, V)
    sd.sd_filter_logits(t, sd.Sampling(it, k, p, mp), *want)
    given = [torch.from_numpy(a).cuda().to(d) for a, d in ((it, torch.float64), (k, torch.int64), (p, torch.float64), (mp, torch.float64))]
    got, side = outputs(M, V), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        for a in got:
            a.zero_()
        torch.cuda.synchronize()
        torch.cuda._sleep(BUSY)
        if as_argument:
            sd.sd_filter_logits(t, sd.Sampling(*given), *got, stream=side)
        else:
            how = sd.Sampling(*given)
            with torch.cuda.stream(side):
                sd.sd_filter_logits(t, how, *got)
            del how
        junk = [torch.full((M,), -1e30, device="cuda") for _ in range(8)]                  # (what takes the dropped arrays' place)
        torch.cuda.synchronize()
        del junk
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_parameters_outlive_a_call_on_another_stream():
    """Arrays from the host, dropped behind a call that has not begun."""
    M, V = 12, 5000
    t, _ = batch(M, V, "f32", 4)
    params = parameters(M, V, 4, "kpm")
    want = outputs(M, V)
    sd.sd_filter_logits(t, sd.Sampling(*params), *want)
    got, side = outputs(M, V), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
    sd.sd_filter_logits(t, sd.Sampling(*params), *got, stream=side)
    junk = [torch.full((M,), -1.0, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    del junk
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_tensors_that_can_be_taken_as_they_are_stay_the_callers():
    it = torch.ones(3, device="cuda")
    how = sd.Sampling(it, np.full(3, 5))
    assert how.inv_temp is it and how.c.inv_temp == it.data_ptr() and how.top_k.dtype == torch.int32
