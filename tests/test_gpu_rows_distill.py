"""GPU: the draft's training loss and its gradient against the 64-bit oracle."""
import os

import numpy as np
import pytest
import torch

from oracle import rows as ref
from paper_2509_18824_b200 import binding as sd
from rows_util import TYPES, device_rows, exact_values

pytestmark = pytest.mark.gpu


def problem(M, V, K, kind, seed, tail, inv_temp, ld=None, twice=True):
    g = np.random.default_rng(seed)
    z = g.normal(size=(M, V)) * 2.0
    for r in range(M):
        at = g.permutation(V)[:min(V, 8)]
        z[r, at] += 12.0 * g.random(at.size)
    if M > 3:
        z[3, (g.random(V) < 0.3) & (np.arange(V) > 0)] = -np.inf  # (one entry is left)
    t = device_rows(z.astype(np.float32), kind, ld)
    z = exact_values(t)
    teacher = np.where(np.isfinite(z), z, 0.0) + 0.5 * g.normal(size=z.shape)
    idx = np.full((M, K), -1, dtype=np.int32)
    val = np.zeros((M, K), dtype=np.float32)
    t_lse = np.empty(M, dtype=np.float32)
    label = g.integers(0, V, M).astype(np.int32)
    for r in range(M):
        allowed = np.where(np.isfinite(z[r]), teacher[r], -np.inf)
        v, i, l = ref.top(allowed, K, inv_temp)
        idx[r], val[r], t_lse[r] = i, np.where(i >= 0, v, 0.0), l
        label[r] = i[0] if r % 3 == 0 else label[r]               # a label among the entries
        while not np.isfinite(z[r, label[r]]):
            label[r] = (label[r] + 1) % V
    idx[g.random((M, K)) < 0.1] = -1
    if twice and K >= 4:
        idx[0, 3] = idx[0, 1]                                     # the same index twice, and three times
        if M > 2:
            idx[2, 1:4] = idx[2, 0]
    if M > 1:
        idx[1] = -1                                               # no entry at all
        label[1] = -1                                             # and no label
    if M > 5:
        label[5] = -1
    dloss = g.uniform(0.2, 2.0, M).astype(np.float32)
    if M > 4:
        dloss[4] = 0.0
    return t, z, val, idx, t_lse if tail else None, label, dloss


def cu(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def loss(t, val, idx, t_lse, label, inv_temp, w, dloss=None, grad=None, want_stats=True, status=0):
    M = t.shape[0]
    kl, ce = torch.full((M,), 7.0, device="cuda"), torch.full((M,), 7.0, device="cuda")
    stats = torch.full((M, 4), 7.0, device="cuda") if want_stats else None
    st = sd.new_status()
    sd.sd_distill_loss(t, cu(val), cu(idx), cu(t_lse), cu(label), inv_temp, w[0], w[1], kl, ce, stats, cu(dloss), grad, st)
    torch.cuda.synchronize()
    assert int(st.item()) == status
    return kl.cpu().numpy(), ce.cpu().numpy(), stats


def grad_alone(t, val, idx, t_lse, label, inv_temp, w, stats, dloss, grad, status=0):
    st = sd.new_status()
    sd.sd_distill_grad(t, cu(val), cu(idx), cu(t_lse), cu(label), inv_temp, w[0], w[1], stats, cu(dloss), grad, st)
    torch.cuda.synchronize()
    assert int(st.item()) == status


def check_rows(kind, z, val, idx, t_lse, label, dloss, inv_temp, w, kl, ce, grads):
    M, V = z.shape
    for r in range(M):
        lab = -1 if label is None else int(label[r])
        k, c, g = ref.distill(z[r], val[r].astype(np.float64), idx[r], None if t_lse is None else float(t_lse[r]), lab, inv_temp, w[0], w[1],
                              1.0 if dloss is None else float(dloss[r]))
        # sums of the row in 32 bits per thread (at most 2^10 terms, each off by 2^-22): 1e-6 of them, so 1e-6 in their logarithm, and one
        # rounding of the result; the parts of kl, of the size of |log p| <= 30, are added in 64 bits
        assert abs(kl[r] - k) <= 2e-6 + 2.0 ** -23 * abs(k), (r, kl[r], k)
        assert abs(ce[r] - c) <= 2e-6 + 2.0 ** -23 * abs(c), (r, ce[r], c)
        # gradient: terms of at most its row's largest factors, each to 2e-6 (exponential of an argument of up to 2^6) plus the sums' 1e-6;
        # and the rounding to the type
        scale = abs(1.0 if dloss is None else float(dloss[r])) * (abs(w[0]) * inv_temp + abs(w[1]))
        step = torch.finfo(TYPES[kind]).eps / 2
        for grad in grads:
            got = exact_values(grad)[r]
            assert np.isfinite(got).all()
            # (an entry's gradient is the difference of its s and p: off by shares of s and p, which 1 bounds; elsewhere by shares of s)
            s = np.exp(z[r] * inv_temp - ref.lse(z[r] * inv_temp)) + np.exp(z[r] - ref.lse(z[r]))
            p = np.zeros(V)
            ok = idx[r] >= 0
            np.add.at(p, idx[r][ok], 1.0)
            # (the label's gradient has dloss * ce_weight taken away: the weight rounded to 32 bits, their product, the difference: 3 * 2^-24)
            bound = step * np.abs(g) + scale * (8e-6 * s + 4e-6 * np.minimum(1.0, p) + 1e-30)
            if lab >= 0:
                bound[lab] += 3 * 2.0 ** -24 * scale
            if t_lse is not None:
                bound += scale * 8e-6 * np.abs(s)                 # the rest's ratio
            assert (np.abs(got - g) <= bound).all(), (r, np.abs(got - g).max(), np.argmax(np.abs(got - g) - bound))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("M,V,K,inv_temp,ld,gld", [(7, 4099, 10, 1.0, 4099, 4099), (7, 4099, 64, 0.5, 4104, 4101), (8, 20000, 128, 1.25, 20003, 20003),
                                                   (1, 300, 4, 1.0, 300, 300), (9, 16, 16, 0.75, 17, 24), (6, 2, 1, 1.0, 2, 2), (6, 1, 1, 1.0, 1, 1),
                                                   (7, 2999, 1024, 1.0, 2999, 2999), (3, 152064, 64, 1.0, 152064, 152064), (150, 777, 20, 1.5, 777, 777)])
def test_loss_and_gradient(kind, tail, M, V, K, inv_temp, ld, gld):
    w = (0.9, 0.3)
    t, z, val, idx, t_lse, label, dloss = problem(M, V, K, kind, M + V + K, tail, inv_temp, ld)
    whole = torch.full((M * gld,), 5.0, dtype=TYPES[kind], device="cuda")
    fused = whole.as_strided((M, V), (gld, 1))
    kl, ce, stats = loss(t, val, idx, t_lse, label, inv_temp, w, dloss, fused)
    apart = torch.full((M * gld,), 5.0, dtype=TYPES[kind], device="cuda").as_strided((M, V), (gld, 1))
    grad_alone(t, val, idx, t_lse, label, inv_temp, w, stats, dloss, apart)
    check_rows(kind, z, val, idx, t_lse, label, dloss, inv_temp, w, kl, ce, [fused, apart])
    if gld > V:                                                   # what lies between the rows is as it was
        gaps = torch.cat([whole[r * gld + V:(r + 1) * gld] for r in range(M)])
        assert (gaps == 5.0).all()
    kl2, ce2, _ = loss(t, val, idx, t_lse, label, inv_temp, w, want_stats=False)
    np.testing.assert_array_equal(kl, kl2)
    np.testing.assert_array_equal(ce, ce2)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_gradient_in_the_logits_place(kind):
    t, z, val, idx, t_lse, label, dloss = problem(9, 5003, 32, kind, 1, True, 1.25)
    w = (1.0, 0.1)
    ref_grad = torch.zeros_like(t)
    _, _, stats = loss(t, val, idx, t_lse, label, 1.25, w, dloss, ref_grad)
    one, two = t.clone(), t.clone()
    loss(one, val, idx, t_lse, label, 1.25, w, dloss, one)
    grad_alone(two, val, idx, t_lse, label, 1.25, w, stats, dloss, two)
    assert torch.equal(one, ref_grad) and torch.equal(two, ref_grad)


def test_without_label_weights_and_with_zero_weights():
    t, z, val, idx, t_lse, label, dloss = problem(7, 3000, 16, "f32", 2, True, 1.0)
    grad = torch.zeros_like(t)
    kl = torch.zeros(7, device="cuda")
    st = sd.new_status()
    sd.sd_distill_loss(t, cu(val), cu(idx), cu(t_lse), None, 1.0, 1.0, 0.1, kl, None, None, None, grad, st)
    torch.cuda.synchronize()
    check_rows("f32", z, val, idx, t_lse, None, None, 1.0, (1.0, 0.1), kl.cpu().numpy(), np.zeros(7), [grad])
    for w in ((0.0, 1.0), (1.0, 0.0)):
        kl, ce, stats = loss(t, val, idx, t_lse, label, 1.0, w, None, grad)
        check_rows("f32", z, val, idx, t_lse, label, None, 1.0, w, kl, ce, [grad])


def test_gradient_is_the_losses_difference():
    V, K = 64, 8
    t, z, val, idx, t_lse, label, _ = problem(1, V, K, "f32", 6, True, 1.25)
    grad = torch.zeros_like(t)
    loss(t, val, idx, t_lse, label, 1.25, (1.0, 0.5), None, grad)
    got = exact_values(grad)[0]
    h = 0.01
    both = np.concatenate([np.tile(z, (V, 1)) + h * np.eye(V), np.tile(z, (V, 1)) - h * np.eye(V)]).astype(np.float32)
    rep = lambda a: np.repeat(a, 2 * V, axis=0)
    kl, ce, _ = loss(device_rows(both, "f32"), rep(val), rep(idx), rep(t_lse), rep(label), 1.25, (1.0, 0.5))
    f = kl.astype(np.float64) + 0.5 * ce
    # central differences: h^2 / 6 times the third derivative (below 2), and the losses' 4e-6 over 2 h
    assert np.abs((f[:V] - f[V:]) / (2 * h) - got).max() <= h * h / 3 + 4e-4


def test_entries_and_labels_outside_the_vocabulary():
    t, z, val, idx, t_lse, label, dloss = problem(6, 1000, 8, "f32", 3, False, 1.0)
    idx[0, 2] = 1000
    label[2] = 5000
    grad = torch.zeros_like(t)
    kl, ce, stats = loss(t, val, idx, t_lse, label, 1.0, (1.0, 1.0), dloss, grad, status=sd.SD_ERR_BOUNDS)
    apart = torch.zeros_like(t)
    grad_alone(t, val, idx, t_lse, label, 1.0, (1.0, 1.0), stats, dloss, apart, status=sd.SD_ERR_BOUNDS)
    idx[0, 2], label[2] = -1, -1
    check_rows("f32", z, val, idx, t_lse, label, dloss, 1.0, (1.0, 1.0), kl, ce, [grad, apart])


def test_weightless_rows_with_nan_have_no_gradient():
    t, z, val, idx, t_lse, label, dloss = problem(6, 1000, 8, "bf16", 3, True, 1.0)
    t[4, ::7] = float("nan")                                      # (weight 0)
    grad = torch.full_like(t, 3.0)
    loss(t, val, idx, t_lse, label, 1.0, (1.0, 1.0), dloss, grad)
    assert (grad[4] == 0).all() and torch.isfinite(grad.float()).all()


def test_repeated_calls_agree():
    t, z, val, idx, t_lse, label, dloss = problem(40, 20000, 64, "bf16", 9, True, 1.0)
    first = torch.zeros_like(t)
    a = loss(t, val, idx, t_lse, label, 1.0, (1.0, 0.1), dloss, first)
    for _ in range(3):
        again = torch.zeros_like(t)
        b = loss(t, val, idx, t_lse, label, 1.0, (1.0, 0.1), dloss, again)
        assert torch.equal(first, again) and (a[0] == b[0]).all() and (a[1] == b[1]).all() and torch.equal(a[2], b[2])


def test_a_copy_that_does_not_come_is_reported(monkeypatch):
    t, z, val, idx, t_lse, label, dloss = problem(2, 3000, 8, "f32", 4, True, 1.0)
    monkeypatch.setenv("SDV_TEST_WAIT_CYCLES", "100000")
    monkeypatch.setenv("SDV_TEST_WITHHOLD", "1")
    loss(t, val, idx, t_lse, label, 1.0, (1.0, 0.1), dloss, torch.zeros_like(t), status=sd.SD_ERR_TIMEOUT)
    monkeypatch.delenv("SDV_TEST_WITHHOLD")
    monkeypatch.delenv("SDV_TEST_WAIT_CYCLES")
    kl, ce, _ = loss(t, val, idx, t_lse, label, 1.0, (1.0, 0.1), dloss, torch.zeros_like(t))
    check_rows("f32", z, val, idx, t_lse, label, dloss, 1.0, (1.0, 0.1), kl, ce, [])


def test_captured_and_replayed():
    """Teacher's rows, loss and gradient captured into a graph and replayed on new logits."""
    M, V, K = 12, 4099, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    teacher, student = (torch.randn((M, V), generator=g, device="cuda") for _ in range(2))
    f, i = (lambda *s: torch.zeros(s, device="cuda")), (lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda"))
    val, idx, lse, kl, ce, grad, st = f(M, K), i(M, K), f(M), f(M), f(M), f(M, V), sd.new_status()

    def step():
        sd.sd_top_logits(teacher, 1.0, val, idx, lse, st)
        sd.sd_distill_loss(student, val, idx, lse, idx[:, 0].contiguous(), 1.0, 1.0, 0.1, kl, ce, None, None, grad, st)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        teacher.normal_(generator=g)
        student.normal_(generator=g)
        graph.replay()
        got = [a.clone() for a in (val, idx, lse, kl, ce, grad)]
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (val, idx, lse, kl, ce, grad)):
            assert torch.equal(a, b)
    assert int(st.item()) == 0


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V,K,inv_temp", [(4099, 16, 1.0), (20000, 40, 0.5), (152064, 64, 1.0), (3001, 427, 1.25)])
def test_the_loss_of_a_draft_that_has_learned(kind, V, K, inv_temp):
    """Small divergences, differences of sums that nearly agree."""
    g = np.random.default_rng(V)
    M = 9
    t = device_rows((g.normal(size=(M, V)) * 3.0).astype(np.float32), kind)
    z = exact_values(t)
    teacher = z + 0.03 * g.normal(size=z.shape)
    idx, val, t_lse = np.zeros((M, K), dtype=np.int32), np.zeros((M, K), dtype=np.float32), np.zeros(M, dtype=np.float32)
    for r in range(M):
        val[r], idx[r], t_lse[r] = ref.top(teacher[r], K, inv_temp)
    kl, _, _ = loss(t, val, idx, t_lse, None, inv_temp, (1.0, 0.0))
    for r in range(M):
        want, _, _ = ref.distill(z[r], val[r].astype(np.float64), idx[r], float(t_lse[r]), -1, inv_temp, 1.0, 0.0)
        s = np.exp(z[r] * inv_temp - ref.lse(z[r] * inv_temp))
        p = np.exp(val[r].astype(np.float64) * inv_temp - float(t_lse[r]))
        s_list = s[idx[r]].sum()
        # kl = .. - sum p log s_k - p_rest log s_rest: the rest's sum is off by 2e-6 of itself (exponentials to 2^-22 and their arguments),
        # which counts by s_rest - p_rest; the entries' are in 64 bits, of a temperature that 32 bits round (2^-24 of the logits' distance
        # from the largest, by s - p); terms of up to 20 to 1e-11; one rounding of the result
        change = np.abs(s[idx[r]] - p).sum() + abs((1 - s_list) - (1 - p.sum()))
        far = inv_temp * (z[r].max() - z[r].min())
        assert abs(kl[r] - want) <= 2e-6 * abs(s_list - p.sum()) + 2.0 ** -24 * far * change + 1e-9 + 2.0 ** -23 * abs(want), (r, kl[r], want)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 4099, 40000])
def test_logits_of_any_size(kind, V):
    """Up to |logit * inv_temp| of 1e8 the losses are those of the formula; beyond, NaN (never a number that is wrong)."""
    g = np.random.default_rng(V)
    K, size = 8, np.array([1e-3, 1.0, 1e3, 1e6, 1e7, 2e9, 1e12, 1e20, 1e37])
    M = size.size
    x = g.normal(size=(M, V))
    x = np.clip(x, -4.0, 4.0) * size[:, None]
    t = device_rows(x.astype(np.float32), kind)
    z = exact_values(t)
    teacher = np.clip(g.normal(size=(M, V)), -4.0, 4.0) * np.minimum(size, 1e7)[:, None]
    for inv_temp in (0.5, 1.0, 1.25):
        idx, val, label = np.zeros((M, K), dtype=np.int32), np.zeros((M, K), dtype=np.float32), g.integers(0, V, M).astype(np.int32)
        for r in range(M):
            val[r], idx[r], _ = ref.top(teacher[r], K, inv_temp)
        grad = torch.zeros_like(t)
        kl, ce, _ = loss(t, val, idx, None, label, inv_temp, (1.0, 0.5), None, grad)
        gr = grad.double().cpu().numpy()
        for r in range(M):
            if size[r] > 1e8:
                assert np.isnan(kl[r]) and np.isnan(ce[r]) and np.isnan(gr[r]).any()
                continue
            a, b, want = ref.distill(z[r], val[r].astype(np.float64), idx[r], None, int(label[r]), inv_temp, 1.0, 0.5)
            # a temperature that 32 bits round (2^-24 of the logits' distance), sums to 2e-6, one rounding
            far = inv_temp * (z[r].max() - z[r].min())
            assert abs(kl[r] - a) <= 2.0 ** -24 * 2 * far + 2e-6 + 2.0 ** -23 * abs(a), (size[r], kl[r], a)
            assert abs(ce[r] - b) <= 2.0 ** -24 * 2 * (z[r].max() - z[r].min()) + 2e-6 + 2.0 ** -23 * abs(b), (size[r], ce[r], b)
            assert np.isfinite(gr[r]).all()
