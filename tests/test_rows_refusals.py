"""Argument checks of the calls on rows of logits: refused on the host, before any launch (no GPU here)."""
import ctypes

import pytest

from paper_2509_18824_b200 import binding as b

f = ctypes.c_float
ok = 4096                                                   # any 16-byte aligned, non-null stand-in address


def top(logits=ok, dtype=0, ld=100, M=4, V=100, K=10, it=1.0, values=ok, index=ok, lse=ok, st=ok):
    return b.lib.sd_top_logits(logits, dtype, ld, M, V, K, f(it), values, index, lse, st, None)


def sample(logits=ok, dtype=0, ld=100, M=4, V=100, how=True, u=ok, N=1, tokens=ok, prob=ok, probs=None, lse=ok, st=ok, params=(ok, ok, ok, ok)):
    c = b.sd_sampling(*params)
    return b.lib.sd_sample_logits(logits, dtype, ld, M, V, ctypes.byref(c) if how else None, u, N, tokens, prob, probs, lse, st, None)


def filt(logits=ok, dtype=0, ld=100, M=4, V=100, out=8192, lse=ok, kept=None, st=ok):
    c = b.sd_sampling(None, None, None, None)
    return b.lib.sd_filter_logits(logits, dtype, ld, M, V, ctypes.byref(c), out, lse, kept, st, None)


def loss(logits=ok, dtype=0, ld=100, M=4, V=100, val=ok, idx=ok, K=10, lse=None, label=ok, it=1.0, kl=ok, ce=ok, stats=None, dloss=None, grad=None, gld=100, st=ok):
    return b.lib.sd_distill_loss(logits, dtype, ld, M, V, val, idx, K, lse, label, f(it), f(1.0), f(0.1), kl, ce, stats, dloss, grad, gld, st, None)


def grad(logits=ok, dtype=0, ld=100, M=4, V=100, val=ok, idx=ok, K=10, it=1.0, stats=ok, g=8192, gld=100, st=ok):
    return b.lib.sd_distill_grad(logits, dtype, ld, M, V, val, idx, K, None, None, f(it), f(1.0), f(0.1), stats, None, g, gld, st, None)


@pytest.mark.parametrize("call", [top, sample, filt, loss, grad])
def test_rows(call):
    assert call(logits=None) == b.SD_ERR_INVALID_ARG
    assert call(logits=4100) == b.SD_ERR_INVALID_ARG
    assert call(st=None) == b.SD_ERR_INVALID_ARG
    assert call(ld=99) == b.SD_ERR_INVALID_ARG
    assert call(V=0) == b.SD_ERR_INVALID_ARG
    assert call(M=-1) == b.SD_ERR_INVALID_ARG
    assert call(dtype=2) == b.SD_ERR_UNSUPPORTED
    assert call(dtype=-1) == b.SD_ERR_UNSUPPORTED
    assert call(V=262145, ld=300000) == b.SD_ERR_UNSUPPORTED
    assert call(M=(1 << 24) + 1) == b.SD_ERR_UNSUPPORTED
    assert call(M=0, logits=None) == b.SD_OK                # nothing to do, nothing launched


def test_top():
    assert top(K=0) == b.SD_ERR_INVALID_ARG
    assert top(K=1025) == b.SD_ERR_UNSUPPORTED
    for it in (0.0, -1.0, float("nan"), float("inf")):
        assert top(it=it) == b.SD_ERR_INVALID_ARG
    for bad in (None, 4098):
        assert top(values=bad) == b.SD_ERR_INVALID_ARG
        assert top(index=bad) == b.SD_ERR_INVALID_ARG
    assert top(lse=4097) == b.SD_ERR_INVALID_ARG


def test_sample():
    assert sample(how=False) == b.SD_ERR_INVALID_ARG
    assert sample(N=0) == b.SD_ERR_INVALID_ARG
    assert sample(N=65) == b.SD_ERR_UNSUPPORTED
    for bad in (None, 4098):
        assert sample(u=bad) == b.SD_ERR_INVALID_ARG
        assert sample(tokens=bad) == b.SD_ERR_INVALID_ARG
    assert sample(prob=4098) == b.SD_ERR_INVALID_ARG
    assert sample(probs=8196) == b.SD_ERR_INVALID_ARG
    assert sample(probs=ok) == b.SD_ERR_INVALID_ARG         # the logits themselves
    for i in range(4):
        assert sample(params=tuple(4098 if j == i else ok for j in range(4))) == b.SD_ERR_INVALID_ARG


def test_filter():
    assert filt(out=None) == b.SD_ERR_INVALID_ARG
    assert filt(out=8196) == b.SD_ERR_INVALID_ARG
    assert filt(lse=None) == b.SD_ERR_INVALID_ARG
    assert filt(kept=4098) == b.SD_ERR_INVALID_ARG
    assert filt(out=ok, dtype=1) == b.SD_ERR_INVALID_ARG    # in place: only f32 rows without gaps
    assert filt(out=ok, ld=101) == b.SD_ERR_INVALID_ARG


def test_distill():
    for call in (loss, grad):
        assert call(K=0) == b.SD_ERR_INVALID_ARG
        assert call(K=1025) == b.SD_ERR_UNSUPPORTED
        for it in (0.0, -1.0, float("nan"), float("inf")):
            assert call(it=it) == b.SD_ERR_INVALID_ARG
        for bad in (None, 4098):
            assert call(val=bad) == b.SD_ERR_INVALID_ARG
            assert call(idx=bad) == b.SD_ERR_INVALID_ARG
    assert loss(kl=None) == b.SD_ERR_INVALID_ARG
    assert loss(ce=None) == b.SD_ERR_INVALID_ARG            # (a label needs it)
    assert loss(stats=8196) == b.SD_ERR_INVALID_ARG
    assert loss(grad=8196) == b.SD_ERR_INVALID_ARG
    assert loss(grad=8192, gld=99) == b.SD_ERR_INVALID_ARG
    assert loss(grad=ok, gld=104) == b.SD_ERR_INVALID_ARG   # in place: the same rows
    assert loss(dloss=4098) == b.SD_ERR_INVALID_ARG
    assert grad(g=None) == b.SD_ERR_INVALID_ARG
    assert grad(stats=None) == b.SD_ERR_INVALID_ARG
    assert grad(stats=8196) == b.SD_ERR_INVALID_ARG
    assert grad(g=ok, gld=104) == b.SD_ERR_INVALID_ARG
