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


def test_parameters_that_are_converted_on_a_busy_side_stream():
    """And read on the default one."""
    M, V = 12, 5000
    t, _ = batch(M, V, "f32", 3)
    params = parameters(M, V, 3, "kpm")
    want = outputs(M, V)
    sd.sd_filter_logits(t, sd.Sampling(*params), *want)
    given = [torch.from_numpy(a).cuda().to(d) for a, d in zip(params, (torch.float64, torch.int64, torch.float64, torch.float64))]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (None, 0, torch.cuda.default_stream()):
        got = outputs(M, V)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(BUSY)
            how = sd.Sampling(*given)
        sd.sd_filter_logits(t, how, *got, stream=stream)
        torch.cuda.synchronize()
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


def test_a_step_s_first_call_on_another_stream():
    """The buffers that the first call makes are not filled behind what it writes."""
    from paper_2509_18824_b200 import workloads as wl
    from paper_2509_18824_b200.step import VerifyStep
    w = wl.make("c5", hidden_gain=12.0, B=3, L=1, V=8192, Hd=128, prefix=100)
    M = w.B * w.T_max
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q = torch.softmax(torch.randn((w.B, w.T_max, w.V), device="cuda", generator=g), dim=-1)
    u, wv = torch.rand((w.B, w.T_max), device="cuda", generator=g), torch.rand(w.B, device="cuda", generator=g)
    how = sd.Sampling(np.full(M, 0.9), np.full(M, 100))
    one, two, side = VerifyStep(w), VerifyStep(w), torch.cuda.Stream()
    one.tail_filtered(how, q, u, wv)
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    two.tail_filtered(how, q, u, wv, stream=side)
    torch.cuda.synchronize()
    for name in ("logits", "lse_filtered", "n_acc", "path", "out_tok", "new_len"):
        assert torch.equal(getattr(one, name), getattr(two, name)), name
