"""GPU: top logits, sampling and filtering of rows of logits against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import rows as ref
from paper_2509_18824_b200 import binding as sd
from rows_util import LOWEST, PATTERNS, TYPES, device_rows, exact_values, margin, row

pytestmark = pytest.mark.gpu

# Borders and draws: masses are off by 1e-11 of themselves, sums of the flat rows' histograms by 2^-44 of the largest mass per
# entry (20000 entries: 1.2e-9); a row within BORDER of a border may fall to either side.
BORDER = 1e-8


def batch(M, V, kind, seed, patterns=PATTERNS, ld=None):
    g = np.random.default_rng(seed)
    x = np.stack([row(patterns[r % len(patterns)], V, g, LOWEST[kind]) for r in range(M)])
    t = device_rows(x.astype(np.float32), kind, ld)
    return t, exact_values(t)


def parameters(M, V, seed, which):
    g = np.random.default_rng(seed + 100)
    it = g.uniform(0.6, 1.6, M).astype(np.float32)
    k = p = mp = None
    if "g" in which:
        it[::5] = np.inf
    if "k" in which:
        k = g.choice([0, 1, 2, 17, 64, 500, 1024, 1025, 3000, V - 1, V], M).astype(np.int32)
    if "p" in which:
        p = g.choice([-0.5, 0.0, 0.3, 0.7, 0.9, 0.99, 0.9999, 1.0, 2.0], M).astype(np.float32)
    if "m" in which:
        mp = g.choice([-1.0, 0.0, 1e-4, 0.05, 0.5, 1.0, 3.0], M).astype(np.float32)
    return it, k, p, mp


def of_row(params, r):
    it, k, p, mp = params
    return dict(inv_temp=float(it[r]), top_k=0 if k is None else int(k[r]), top_p=1.0 if p is None else float(p[r]), min_p=0.0 if mp is None else float(mp[r]))


def sample(t, params, u, probs=True, how=None):
    M, V = t.shape
    N = u.shape[1]
    tokens = torch.full((M, N), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((M, N), 7.0, device="cuda")
    dense = torch.full((M, V), 7.0, device="cuda") if probs else None
    lse = torch.full((M,), 7.0, device="cuda")
    st = sd.new_status()
    sd.sd_sample_logits(t, how or sd.Sampling(*params), torch.from_numpy(u).cuda(), tokens, prob, dense, lse, st)
    torch.cuda.synchronize()
    return tokens.cpu().numpy(), prob.cpu().numpy(), None if dense is None else dense.cpu().numpy(), lse.cpu().numpy(), int(st.item())


def filtered(t, params, out=None):
    M, V = t.shape
    out = torch.full((M, V), 7.0, device="cuda") if out is None else out
    lse = torch.full((M,), 7.0, device="cuda")
    kept = torch.full((M,), -7, dtype=torch.int32, device="cuda")
    st = sd.new_status()
    sd.sd_filter_logits(t, sd.Sampling(*params), out, lse, kept, st)
    torch.cuda.synchronize()
    return out.cpu().numpy(), lse.cpu().numpy(), kept.cpu().numpy(), int(st.item())


def close(got, want, rel, abs_=0.0):
    """got (f32 outputs) against want: infinities alike, else within rel of the value and abs_."""
    want = np.asarray(want, dtype=np.float64)
    np.testing.assert_array_equal(np.isfinite(got), np.isfinite(want))
    f = np.isfinite(want)
    np.testing.assert_array_equal(np.asarray(got, dtype=np.float64)[~f], want[~f])
    assert (np.abs(got[f] - want[f]) <= rel * np.abs(want[f]) + abs_).all()


def check(t, x, params, seed, N=3, probs=True, decisive=0.9):
    M, V = x.shape
    u = np.random.default_rng(seed).random((M, N)).astype(np.float32)
    u[0, 0] = 0.0
    u[-1, -1] = np.float32(1 - 2 ** -24)
    tokens, prob, dense, lse, st = sample(t, params, u, probs)
    out, flse, kept, fst = filtered(t, params)
    assert st == 0 and fst == 0
    decided = 0
    for r in range(M):
        how = of_row(params, r)
        if margin(x[r], **how) < BORDER:
            continue
        o, z = ref.keep(x[r], **how)
        p = ref.probabilities(x[r], **how)
        assert kept[r] == o.size, (r, how)
        stays = np.zeros(V, dtype=bool)
        stays[o] = True
        # scaled logits: one rounding of the product; lse: one of the result
        close(out[r], np.where(stays, z, -np.inf), 2.0 ** -24)
        want_lse = ref.lse(z[o]) if o.size else -np.inf
        close(lse[r:r + 1], [want_lse], 2.0 ** -23, 1e-9)
        close(flse[r:r + 1], [want_lse], 2.0 ** -23, 1e-9)
        if dense is not None:
            # 2^(d c) with d c rounded twice (d <= 64 factors of two where p matters: 64 * 2^-23 ln 2), its factor, the function
            close(dense[r], p, 8e-6, 1e-24)
        for n in range(N):
            want, far = ref.draw(p, float(u[r, n]))
            if far < BORDER and o.size > 1:
                continue
            decided += 1
            assert tokens[r, n] == want, (r, n, how)
            assert prob[r, n] == pytest.approx(p[want] if want >= 0 else 0.0, rel=2.0 ** -22)
    assert decided >= decisive * M * N


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,which", [(26, 4099, "kpm"), (26, 4099, "kg"), (26, 20000, "p"), (13, 20000, "m"), (13, 20000, ""), (26, 20000, "kp"),
                                       (39, 257, "kpm"), (13, 1, "kpm"), (13, 7, "pm"), (1, 20000, "kpm"), (2, 152064, "p"), (13, 152064, "kpmg")])
def test_sampling_and_filter(kind, M, V, which):
    t, x = batch(M, V, kind, M + V)
    check(t, x, parameters(M, V, M + V, which), V)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("V,ld", [(4099, 4101), (20000, 20003), (33, 50)])
def test_rows_apart_and_at_any_place(kind, V, ld):
    t, x = batch(26, V, kind, ld, ld=ld)
    check(t, x, parameters(26, V, ld, "kpm"), ld)


@pytest.mark.parametrize("M", [149, 400])
def test_many_rows(M):
    t, x = batch(M, 5001, "f32", M)
    check(t, x, parameters(M, 5001, M, "kpmg"), M, N=1)


@pytest.mark.parametrize("N", [1, 17, 64])
def test_many_draws_of_a_row(N):
    t, x = batch(13, 20000, "f32", N)
    check(t, x, parameters(13, 20000, N, "p"), N, N=N, probs=False)


def test_largest_vocabulary():
    t, x = batch(13, 262144, "f32", 5)
    check(t, x, parameters(13, 262144, 5, "kpm"), 5, N=2)


def test_filter_in_place_and_repeated_calls_agree():
    t, x = batch(39, 4099, "f32", 8)
    params = parameters(39, 4099, 8, "kpm")
    first = filtered(t, params)
    for _ in range(3):
        again = filtered(t, params)
        for a, b in zip(first, again):
            np.testing.assert_array_equal(a, b)
    copy = t.clone()
    into = filtered(copy, params, out=copy)
    for a, b in zip(first, into):
        np.testing.assert_array_equal(a, b)


def test_bad_numbers_are_reported_row_by_row():
    t, x = batch(6, 1000, "f32", 2, patterns=("bulk",))
    it = np.array([1.0, 0.0, -1.0, np.nan, 1e-7, 1.0], dtype=np.float32)
    u = np.full((6, 2), 0.5, dtype=np.float32)
    tokens, prob, dense, lse, st = sample(t, (it, None, None, None), u)
    assert st == sd.SD_ERR_INVALID_ARG
    assert (tokens[1:5] == -1).all() and (prob[1:5] == 0).all() and (dense[1:5] == 0).all() and np.isneginf(lse[1:5]).all()
    assert (tokens[[0, 5]] >= 0).all()
    for how in ((None, [5] * 6, None, None), (None, None, None, None)):
        u = np.array([[0.5, 1.0], [-0.1, 0.5], [np.nan, 0.5], [0.5, np.inf], [0.5, 0.5], [0.0, 0.9]], dtype=np.float32)
        tokens, prob, _, _, st = sample(t, how, u)
        assert st == sd.SD_ERR_INVALID_ARG
        good = (u >= 0) & (u < 1)
        assert (tokens[good] >= 0).all() and (tokens[~good] == -1).all() and (prob[~good] == 0).all()


def test_no_parameters_at_all_is_the_row_s_own_distribution():
    t, x = batch(13, 3000, "bf16", 4)
    ones = np.ones(13, dtype=np.float32)
    u = np.random.default_rng(0).random((13, 2)).astype(np.float32)
    a = sample(t, (None, None, None, None), u)
    b = sample(t, (ones, None, None, None), u)
    for p, q in zip(a, b):
        np.testing.assert_array_equal(p, q)


def test_no_rows():
    t = torch.empty((0, 100), device="cuda")
    st = sd.new_status()
    f, i = (lambda *s: torch.empty(s, device="cuda")), (lambda *s: torch.empty(s, dtype=torch.int32, device="cuda"))
    sd.sd_sample_logits(t, sd.Sampling(), f(0, 2), i(0, 2), None, None, None, st)
    sd.sd_filter_logits(t, sd.Sampling(), f(0, 100), f(0), None, st)
    sd.sd_top_logits(t, 1.0, f(0, 4), i(0, 4), None, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0


# ---------------------------------------------------------------------------------------------- top logits
def top(t, K, inv_temp):
    M, V = t.shape
    values = torch.full((M, K), 7.0, device="cuda")
    index = torch.full((M, K), -7, dtype=torch.int32, device="cuda")
    lse = torch.full((M,), 7.0, device="cuda")
    st = sd.new_status()
    sd.sd_top_logits(t, inv_temp, values, index, lse, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    return values.cpu().numpy(), index.cpu().numpy(), lse.cpu().numpy()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K,ld", [(13, 4099, 10, 4099), (26, 4099, 1024, 4103), (13, 20000, 64, 20000), (1, 20000, 1, 20000), (13, 20000, 600, 20001),
                                      (13, 5, 12, 9), (13, 1, 1, 1), (13, 152064, 128, 152064), (170, 3001, 33, 3001), (300, 20000, 257, 20000)])
def test_top_logits(kind, M, V, K, ld):
    t, x = batch(M, V, kind, K, ld=ld)
    values, index, lse = top(t, K, 0.8)
    for r in range(M):
        v, i, l = ref.top(x[r], K, float(np.float32(0.8)))
        np.testing.assert_array_equal(index[r], i, err_msg=str(r))
        np.testing.assert_array_equal(values[r].astype(np.float64) + 0.0, v + 0.0)
        # sums of V terms that are off by 2^-22 and an argument of at most 2^6 rounded to 2^-24 of it each, in 32 bits
        assert lse[r] == l if np.isinf(l) else abs(lse[r] - l) <= 2e-5 + 2.0 ** -23 * abs(l)


def test_top_logits_with_infinity():
    x = np.zeros((2, 500), dtype=np.float32)
    x[0, 7] = np.inf
    x[1, 3] = -np.inf
    values, index, lse = top(device_rows(x, "f32"), 3, 1.0)
    assert index.tolist() == [[7, 0, 1], [0, 1, 2]] and values[0, 0] == np.inf
    assert lse[0] == np.inf and lse[1] == pytest.approx(np.log(499), rel=1e-6)
