"""GPU: rows of logits in numbers at which a call reads them from memory more than once (or in shares of one, two and four CTAs), in
place, in graphs and on two streams; copies that do not come."""
import numpy as np
import pytest
import torch

from oracle import rows as ref
from paper_2509_18824_b200 import binding as sd
from rows_util import LOWEST, device_rows, exact_values, margin
from test_gpu_rows_sampling import BORDER, batch, check, filtered, of_row, parameters, sample, top

pytestmark = pytest.mark.gpu


# 152064 f32 of 40 to 74 rows: shares of a quarter; fewer than 297 rows: halves; beyond: whole rows (20600 f32 and 41000 bf16 are more than
# a CTA's shared memory holds)
@pytest.mark.parametrize("kind,M,V,ld,which", [("f32", 80, 41000, 41000, "kpm"), ("f32", 80, 41001, 41007, "p"), ("f32", 160, 20600, 20600, "kpmg"),
                                               ("f32", 160, 20603, 20603, ""), ("f32", 900, 20600, 20601, "kpm"), ("f32", 80, 41000, 41000, "m"),
                                               ("f32", 52, 152064, 152064, "kpm"), ("f32", 39, 152065, 152069, "p"), ("f32", 74, 82001, 82001, "m"), ("bf16", 74, 262143, 262144, "kpmg"),
                                               ("bf16", 80, 82001, 82001, "kpm"), ("bf16", 160, 41000, 41000, "p"), ("bf16", 900, 41100, 41100, "kpmg"),
                                               ("bf16", 160, 41003, 41011, "kp")])
def test_many_rows(kind, M, V, ld, which):
    t, x = batch(M, V, kind, M + V, ld=ld)
    check(t, x, parameters(M, V, M + V, which), M, N=1)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_flat_rows_of_the_largest_vocabulary(kind):
    """All mass in a few bins of a histogram, in a single one even: sums that 32 bits hold only in parts."""
    M, V = 76, 262144
    t, x = batch(M, V, kind, 3, patterns=("equal", "flat", "all_lowest", "bulk", "rising"))
    it = np.ones(M, dtype=np.float32)
    p = np.resize(np.array([0.5, 0.9, 0.999], dtype=np.float32), M)
    k = np.resize(np.array([0, 0, 0, 0, 200000, 1500], dtype=np.int32), M)
    # (equal logits at p = 0.5 have a border at exactly half of the entries: two patterns in five, one row in three, are left out)
    check(t, x, (it, k, p, None), 1, N=1, decisive=1 - 2 / 15 - 0.05)


@pytest.mark.parametrize("M,V", [(45, 100003), (80, 41000), (160, 20603), (900, 20600)])
def test_filter_in_place_and_repeated(M, V):
    t, x = batch(M, V, "f32", 8)
    params = parameters(M, V, 8, "kpm")
    first = filtered(t, params)
    again = filtered(t, params)
    copy = t.clone()
    into = filtered(copy, params, out=copy)
    for a, b, c in zip(first, again, into):
        np.testing.assert_array_equal(a, b)
        np.testing.assert_array_equal(a, c)


def test_shares_of_a_row_do_not_change_what_stays():
    """The same rows in calls of 20, 40, 80 and 400 rows."""
    V = 90001
    t, x = batch(20, V, "f32", 21)
    params = parameters(20, V, 21, "kpm")
    u = np.random.default_rng(2).random((20, 2)).astype(np.float32)
    want = sample(t, params, u)
    out = filtered(t, params)
    for times in (2, 4, 20):
        many = t.repeat(times, 1)
        tiled = tuple(None if a is None else np.tile(a, times) for a in params)
        tokens, prob, dense, lse, st = sample(many, tiled, np.tile(u, (times, 1)))
        o, l, kept, fst = filtered(many, tiled)
        assert st == 0 and fst == 0
        for i in range(times):
            s = slice(i * 20, i * 20 + 20)
            np.testing.assert_array_equal(tokens[s], want[0])
            np.testing.assert_array_equal(kept[s], out[2])
            np.testing.assert_array_equal(o[s], out[0])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K,ld", [(80, 20000, 112, 20000), (80, 20000, 113, 20007), (149, 9001, 300, 9001), (149, 9001, 384, 9003), (149, 9001, 385, 9001),
                                      (300, 700, 384, 701), (300, 50, 200, 50), (74, 3, 3, 3)])
def test_top_logits_of_many_rows(kind, M, V, K, ld):
    t, x = batch(M, V, kind, K, ld=ld)
    values, index, lse = top(t, K, 1.25)
    for r in range(M):
        v, i, l = ref.top(x[r], K, 1.25)
        np.testing.assert_array_equal(index[r], i, err_msg=str(r))
        np.testing.assert_array_equal(values[r].astype(np.float64) + 0.0, v + 0.0)
        # sums of V terms that are off by 2^-22 and an argument of at most 2^6 rounded to 2^-24 of it each, in 32 bits
        assert lse[r] == l if np.isinf(l) else abs(lse[r] - l) <= 2e-5 + 2.0 ** -23 * abs(l)


def calls(t, M, V, how, u):
    """The three calls on t, as a function that enqueues them on the current stream, and what they write."""
    f, i = (lambda *s: torch.zeros(s, device="cuda")), (lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda"))
    out = dict(values=f(M, 20), index=i(M, 20), top_lse=f(M), tokens=i(M, 2), prob=f(M, 2), probs=f(M, V), lse=f(M), rows=f(M, V), flse=f(M), kept=i(M), st=sd.new_status())

    def enqueue():
        st = out["st"]
        sd.sd_top_logits(t, 1.0, out["values"], out["index"], out["top_lse"], st)
        sd.sd_sample_logits(t, how, u, out["tokens"], out["prob"], out["probs"], out["lse"], st)
        sd.sd_filter_logits(t, how, out["rows"], out["flse"], out["kept"], st)
    return enqueue, out


@pytest.mark.parametrize("M,V", [(6, 30000), (80, 41000)])
def test_calls_in_a_graph_on_new_rows_and_parameters(M, V):
    t, _ = batch(M, V, "f32", 5)
    how = sd.Sampling(*parameters(M, V, 5, "kpm"))
    u = torch.rand((M, 2), device="cuda")
    enqueue, out = calls(t, M, V, how, u)
    enqueue()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        enqueue()
    for seed in (6, 7):
        t.copy_(batch(M, V, "f32", seed)[0])
        new = sd.Sampling(*parameters(M, V, seed, "kpm"))
        for a, b in ((how.inv_temp, new.inv_temp), (how.top_k, new.top_k), (how.top_p, new.top_p), (how.min_p, new.min_p)):
            a.copy_(b)
        u.uniform_()
        u.clamp_(max=0.9999999)
        graph.replay()
        got = {k: v.clone() for k, v in out.items()}
        for v in out.values():
            v.zero_()
        enqueue()
        torch.cuda.synchronize()
        for k in got:
            assert torch.equal(got[k], out[k]), k
    assert int(out["st"].item()) == 0


def test_two_streams_at_once():
    """Calls of few and of many rows side by side: nothing is shared between them."""
    jobs = []
    for M, V, seed in ((6, 152064, 11), (80, 41000, 12)):
        t, _ = batch(M, V, "f32", seed)
        jobs.append((calls(t, M, V, sd.Sampling(*parameters(M, V, seed, "kpm")), torch.rand((M, 2), device="cuda").clamp_(max=0.9999999)), torch.cuda.Stream()))
    want = []
    for (enqueue, out), _ in jobs:
        enqueue()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in out.items()})
        for v in out.values():
            v.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for (enqueue, out), s in jobs:
            with torch.cuda.stream(s):
                enqueue()
    torch.cuda.synchronize()
    for ((_, out), _), w in zip(jobs, want):
        for k in w:
            assert torch.equal(out[k], w[k]), k
        assert int(out["st"].item()) == 0


def test_a_copy_that_does_not_come_is_reported(monkeypatch):
    M, V = 4, 30000
    t, x = batch(M, V, "f32", 9, patterns=("bulk", "peaks"))
    params = parameters(M, V, 9, "kp")
    u = np.full((M, 1), 0.5, dtype=np.float32)
    monkeypatch.setenv("SDV_TEST_WAIT_CYCLES", "100000")
    monkeypatch.setenv("SDV_TEST_WITHHOLD", "1")
    assert sample(t, params, u)[4] == sd.SD_ERR_TIMEOUT
    assert filtered(t, params)[3] == sd.SD_ERR_TIMEOUT
    values, index, st = torch.zeros((M, 8), device="cuda"), torch.zeros((M, 8), dtype=torch.int32, device="cuda"), sd.new_status()
    sd.sd_top_logits(t, 1.0, values, index, None, st)
    torch.cuda.synchronize()
    assert int(st.item()) == sd.SD_ERR_TIMEOUT
    monkeypatch.delenv("SDV_TEST_WITHHOLD")
    monkeypatch.delenv("SDV_TEST_WAIT_CYCLES")
    check(t, x, params, 9, N=1)


@pytest.mark.parametrize("M,V", [(6, 30000), (45, 100003)])
def test_rows_with_infinity_are_reported_and_the_others_drawn(M, V):
    t, x = batch(M, V, "f32", 13, patterns=("bulk", "peaks", "flat"))
    t[1, 17] = np.inf
    t[2, V - 1] = np.inf
    t[2, 5] = np.inf
    for which in ("kpm", "k", "p", "m", ""):
        params = parameters(M, V, 13, which)
        u = np.random.default_rng(1).random((M, 2)).astype(np.float32)
        tokens, prob, dense, lse, st = sample(t, params, u)
        out, flse, kept, fst = filtered(t, params)
        assert st == sd.SD_ERR_INVALID_ARG and fst == sd.SD_ERR_INVALID_ARG
        assert (tokens[1:3] == -1).all() and (prob[1:3] == 0).all() and (dense[1:3] == 0).all() and np.isneginf(lse[1:3]).all()
        assert np.isneginf(out[1:3]).all() and np.isneginf(flse[1:3]).all() and (kept[1:3] == 0).all()
        rest = [r for r in range(M) if r not in (1, 2)]
        for r in rest:
            how = of_row(params, r)
            if margin(x[r], **how) < BORDER:
                continue
            assert kept[r] == ref.keep(x[r], **how)[0].size
            assert (tokens[r] >= 0).all() and np.isfinite(out[r, tokens[r]]).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_rows_beyond_offsets_of_32_bits(kind):
    """The last rows of 2.3e9 logits end as they do in a call of their own (distillation: to its roundings)."""
    M, V, n, K = 15200, 152064, 8, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    t = torch.empty((M, V), dtype=torch.float32 if kind == "f32" else torch.bfloat16, device="cuda")
    t[:1000].normal_(generator=g)
    for at in range(1000, M, 1000):
        t[at:at + 1000] = t[:min(1000, M - at)]
    t[-n:].normal_(generator=g)
    tail = t[-n:].clone()
    f, i = (lambda *s: torch.zeros(s, device="cuda")), (lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda"))
    res = []
    for x in (t, tail):
        rows = x.shape[0]
        st = sd.new_status()
        values, index, tokens, out, flse, kept, kl, ce = f(rows, K), i(rows, K), i(rows, 1), f(rows, V), f(rows), i(rows), f(rows), f(rows)
        u = torch.full((rows, 1), 0.37, device="cuda")
        how = sd.Sampling(None, torch.full((rows,), 40), None, None)
        sd.sd_top_logits(x, 1.0, values, index, None, st)
        sd.sd_sample_logits(x, how, u, tokens, None, None, None, st)
        sd.sd_filter_logits(x, how, out, flse, kept, st)
        grad = torch.zeros_like(x)
        sd.sd_distill_loss(x, values, index, None, index[:, 3].contiguous(), 1.0, 1.0, 0.5, kl, ce, None, None, grad, st)
        torch.cuda.synchronize()
        assert int(st.item()) == 0
        res.append([a[-n:].clone() for a in (values, index, tokens, out, kept, kl, ce, grad.float())])
        del out, grad
    for a, b in zip(res[0][:5], res[1][:5]):
        assert torch.equal(a, b)
    # two orders of summing 152064 exponentials in 32 bits, then (bf16) a rounding of the gradient each
    for a, b in zip(res[0][5:7], res[1][5:7]):
        assert (a - b).abs().max() <= 4e-6 + 2.0 ** -22 * b.abs().max()
    assert ((res[0][7] - res[1][7]).abs() <= 8e-6 * (res[1][7].abs() + 1e-3) + (2.0 ** -7 * res[1][7].abs() if kind == "bf16" else 0)).all()


@pytest.mark.parametrize("M,V", [(12, 20000), (45, 100003), (320, 20600)])
@pytest.mark.parametrize("which", ["kpm", "p", "m", ""])
def test_extreme_temperatures_and_logits(M, V, which):
    """Exponents far beyond what a mass can have, in every part of the range: distributions of the nearest ones, or flat ones."""
    t, _ = batch(M, V, "f32", 31, patterns=("bulk", "peaks", "equal", "lowest", "all_lowest"))
    it, k, p, mp = parameters(M, V, 31, which)
    it = np.resize(np.array([1e-6, 1.0, 1e5, 1e9, 1e30, 3e38, np.inf], dtype=np.float32), M)
    scale = np.resize(np.array([1.0, 1e6, 1e30], dtype=np.float32), M)
    x = t.cpu().numpy()
    with np.errstate(over="ignore"):
        x = np.clip(x * scale[:, None], LOWEST["f32"], -LOWEST["f32"])
    t.copy_(torch.from_numpy(x))
    x = x.astype(np.float64)
    u = np.random.default_rng(5).random((M, 2)).astype(np.float32)
    tokens, prob, dense, lse, st = sample(t, (it, k, p, mp), u)
    out, flse, kept, fst = filtered(t, (it, k, p, mp))
    assert st == 0 and fst == 0
    decided = 0
    for r in range(M):
        how = of_row((it, k, p, mp), r)
        # the oracle's scaled logits stop at f32's range, which is not where masses come from: relative ones here
        top = x[r].max()
        with np.errstate(over="ignore"):
            rel = np.where(x[r] - top > -1e38, x[r] - top, -1e38)
        if margin(rel, **how) < BORDER:
            continue
        o, z = ref.keep(rel, **how)
        assert kept[r] == o.size, (r, how)
        stays = np.zeros(V, dtype=bool)
        stays[o] = True
        np.testing.assert_array_equal(np.isfinite(out[r]), stays)
        q = ref.probabilities(rel, **how)
        assert (np.abs(dense[r] - q) <= 1e-5 * q + 1e-24).all(), (r, how)
        for n in range(2):
            want, far = ref.draw(q, float(u[r, n]))
            if far >= BORDER or o.size == 1:
                decided += 1
                assert tokens[r, n] == want, (r, n, how)
    assert decided >= M


@pytest.mark.parametrize("which", ["", "p", "kp", "m"])
@pytest.mark.parametrize("kind,M,V", [("f32", 45, 100003), ("bf16", 310, 41111)])
def test_many_draws_of_many_rows(kind, M, V, which):
    t, x = batch(M, V, kind, 41)
    check(t, x, parameters(M, V, 41, which), 41, N=64, probs=False)


@pytest.mark.parametrize("M,V", [(5, 30001), (80, 41000)])
def test_small_arrays_at_any_place_and_outputs_left_out(M, V):
    """The arrays with a few values per row need the alignment of their elements only; what may be missing is."""
    t, x = batch(M, V, "f32", 51)
    params = parameters(M, V, 51, "kpm")
    u = np.random.default_rng(1).random((M, 3)).astype(np.float32)
    want = sample(t, params, u)
    kept_rows = filtered(t, params)

    def odd(a):
        whole = torch.full((a.numel() + 2,), 7, dtype=a.dtype, device="cuda")
        whole[1:-1] = a.reshape(-1)
        return whole, whole[1:-1].view(a.shape)
    how = sd.Sampling(*params)
    for name in ("inv_temp", "top_k", "top_p", "min_p"):
        setattr(how, name, odd(getattr(how, name))[1])
    how.c = sd.sd_sampling(how.inv_temp.data_ptr(), how.top_k.data_ptr(), how.top_p.data_ptr(), how.min_p.data_ptr())
    ut = odd(torch.from_numpy(u).cuda())[1]
    st = sd.new_status()
    tokens_at, tokens = odd(torch.zeros((M, 3), dtype=torch.int32, device="cuda"))
    prob_at, prob = odd(torch.zeros((M, 3), device="cuda"))
    lse_at, lse = odd(torch.zeros(M, device="cuda"))
    sd.sd_sample_logits(t, how, ut, tokens, prob, None, lse, st)
    only = torch.zeros((M, 3), dtype=torch.int32, device="cuda")
    sd.sd_sample_logits(t, how, ut, only, None, None, None, st)
    out = torch.empty((M, V), device="cuda")
    flse_at, flse = odd(torch.zeros(M, device="cuda"))
    sd.sd_filter_logits(t, how, out, flse, None, st)
    values_at, values = odd(torch.zeros((M, 5), device="cuda"))
    index_at, index = odd(torch.zeros((M, 5), dtype=torch.int32, device="cuda"))
    sd.sd_top_logits(t, 1.0, values, index, None, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for got, expect in ((tokens, want[0]), (prob, want[1]), (lse, want[3]), (only, want[0]), (out, kept_rows[0]), (flse, kept_rows[1])):
        np.testing.assert_array_equal(got.cpu().numpy(), expect)
    v, i, _ = top(t, 5, 1.0)
    np.testing.assert_array_equal(index.cpu().numpy(), i)
    np.testing.assert_array_equal(values.cpu().numpy(), v)
    for whole in (tokens_at, prob_at, lse_at, flse_at, values_at, index_at):                # nothing beside them is written
        assert float(whole[0]) == 7 and float(whole[-1]) == 7


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,K", [(3, 60000, 64), (76, 60001, 64), (149, 20000, 300), (149, 60000, 10), (330, 30011, 384)])
def test_top_logits_that_stand_side_by_side(M, V, K, kind):
    """Vocabularies with their frequent tokens at one end: rows that fall, rise, or have a high stretch."""
    g = np.random.default_rng(M + K)
    at = np.arange(V) / V
    shapes = (12.0 * (1 - at), 12.0 * at, 8.0 * np.exp(-at * 50), np.where(np.abs(at - 0.4) < 0.02, 9.0, 0.0), 40.0 * at)
    x = np.stack([g.normal(size=V) * 2.0 + shapes[r % 5] for r in range(M)])
    x[4::10] = np.sort(x[4::10], axis=1)
    t = device_rows(x.astype(np.float32), kind)
    x = exact_values(t)
    values, index, lse = top(t, K, 1.0)
    for r in range(M):
        v, i, l = ref.top(x[r], K, 1.0)
        np.testing.assert_array_equal(index[r], i, err_msg=str(r))
        np.testing.assert_array_equal(values[r].astype(np.float64), v)
        # as above: terms to 2^-22, arguments of at most 2^6 to 2^-24 of them
        assert abs(lse[r] - l) <= 2e-5 + 2.0 ** -23 * abs(l)
    params = (np.ones(M, np.float32), np.resize([50, 5, 0], M).astype(np.int32), np.resize([1.0, 0.9], M).astype(np.float32), None)
    check(t, x, params, 3, N=1)
