"""GPU: the calls on rows of logits from several host threads, whose shared memory differs from call to call."""
import threading

import numpy as np
import pytest
import torch

from paper_2509_18824_b200 import binding as sd

pytestmark = pytest.mark.gpu
LARGE, SMALL = 152064, 4100


def on_a_thread(work):
    """work() on a thread of its own; what it raises is raised here."""
    raised = []

    def body():
        try:
            torch.cuda.set_device(0)
            work()
        except BaseException as e:                            # noqa: B902 (handed on)
            raised.append(e)
    t = threading.Thread(target=body)
    t.start()
    t.join()
    if raised:
        raise raised[0]


def call_of(name, V, K=8):
    """A call on three rows of V logits as a function that makes it, and what it leaves."""
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    M = 3
    x = torch.randn((M, V), device="cuda", generator=g)
    f, i = (lambda *s: torch.zeros(s, device="cuda")), (lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda"))
    st, u, how = sd.new_status(), torch.full((M, 1), 0.4, device="cuda"), sd.Sampling(np.full(M, 0.9), np.full(M, 50), np.full(M, 0.95))
    values, index, lse, out, tokens, kl, grad = f(M, K), i(M, K), f(M), f(M, V), i(M, 1), f(M), f(M, V)
    teacher = (torch.zeros((M, K), device="cuda"), torch.arange(K, device="cuda", dtype=torch.int32).repeat(M, 1), None, None, 1.0, 1.0, 0.0)
    calls = {
        "top": (lambda: sd.sd_top_logits(x, 1.0, values, index, lse, st), (values, index, lse)),
        "sample": (lambda: sd.sd_sample_logits(x, how, u, tokens, None, None, lse, st), (tokens, lse)),
        "filter": (lambda: sd.sd_filter_logits(x, how, out, lse, None, st), (out, lse)),
        "loss": (lambda: sd.sd_distill_loss(x, *teacher, kl, None, None, None, None, st), (kl,)),
        "both": (lambda: sd.sd_distill_loss(x, *teacher, kl, None, None, None, grad, st), (kl, grad)),
    }
    call, left = calls[name]
    return call, left, st


@pytest.mark.parametrize("name", ["top", "sample", "filter", "loss", "both"])
def test_a_small_call_on_another_thread_leaves_the_large_ones_as_they_are(name):
    K = 1024 if name in ("loss", "both") else 8               # (the loss's shared memory goes by K)
    large, left, st = call_of(name, LARGE, K)
    small, _, small_st = call_of(name, SMALL)
    large()
    want = [a.clone() for a in left]
    for a in left:
        a.zero_()
    on_a_thread(small)
    large()
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and int(small_st.item()) == 0
    for a, b in zip(left, want):
        assert torch.equal(a, b)


def test_threads_at_once():
    jobs = [call_of(name, V) for name in ("top", "sample", "filter", "both") for V in (SMALL, 30001, LARGE)]
    want = []
    for call, left, _ in jobs:
        call()
        torch.cuda.synchronize()
        want.append([a.clone() for a in left])

    def many(call):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(50):
                call()
            torch.cuda.current_stream().synchronize()
    raised, threads = [], []
    for call, _, _ in jobs:
        def body(call=call):
            try:
                many(call)
            except BaseException as e:                        # noqa: B902
                raised.append(e)
        threads.append(threading.Thread(target=body))
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not raised, raised
    for (_, left, st), w in zip(jobs, want):
        assert int(st.item()) == 0
        for a, b in zip(left, w):
            assert torch.equal(a, b)
