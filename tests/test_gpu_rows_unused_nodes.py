"""GPU: verification against the filtered target where sequences use fewer nodes than their slots: whatever stands in the slots behind them
(hidden states, sampling parameters, parents, tokens, uniforms, draft distributions) must not matter, and is not reported."""
import numpy as np
import pytest
import torch

from paper_2509_18824_b200 import binding as sd
from paper_2509_18824_b200.step import VerifyStep, to_device
from test_gpu_rows_run import drafts, log_rows, target_parameters, target_rows
from test_gpu_rows_sampling import batch, filtered, parameters, sample
from test_gpu_sampled import decisive_tree_inputs
from test_gpu_sampled_unused_nodes import NODES, junk, ragged

pytestmark = pytest.mark.gpu


def test_sampled_trees_against_the_filtered_target():
    w = ragged("c5", depth=6, L=1)
    B, T = w.B, w.T_max
    M = B * T
    params = target_parameters(M)
    clean = VerifyStep(w)
    p64, x = target_rows(clean, params)
    most = max(int(np.bincount(w.parents[b][1:n], minlength=1).max()) if n > 1 else 1 for b, n in enumerate(NODES))
    probs, tokens, _ = drafts(w, x, 5, most, "f32")
    tok = np.zeros((B, T), dtype=np.int32)
    for b, n in enumerate(NODES):
        seen = np.zeros(T, dtype=int)
        for j in range(1, n):
            i = int(w.parents[b][j])
            tok[b, j] = tokens[b * T + i, seen[i]]
            seen[i] += 1
    q_rows = probs.view(B, T, -1)
    u, wv, ref_n, ref_path, ref_out, _ = decisive_tree_inputs(w, tok, q_rows.cpu().numpy(), log_rows(p64), 1.0, np.random.default_rng(6))
    junk(w, tok, u)
    w.draft_tok = tok
    vs = VerifyStep(w)
    params = [np.array(a) for a in params]
    junk_it = np.resize(np.array([0.0, np.nan, -1.0, np.inf, 1e-9], dtype=np.float32), M)
    for b, n in enumerate(NODES):
        rows = slice(b * T + n, (b + 1) * T)
        params[0][rows] = junk_it[rows]
        params[2][rows] = np.nan
        hidden = vs.hidden.view(torch.bfloat16)
        hidden[rows] = float("inf")
        hidden[rows, ::2] = float("nan")
        q_rows[b, n:] = float("nan")
    how = sd.Sampling(*params)
    for _ in range(2):
        vs.tail_filtered(how, q_rows, to_device(u), to_device(wv))
        torch.cuda.synchronize()
        vs.check_status()
        np.testing.assert_array_equal(vs.n_acc.cpu().numpy(), ref_n)
        np.testing.assert_array_equal(vs.path.cpu().numpy(), ref_path)
        np.testing.assert_array_equal(vs.out_tok.cpu().numpy(), ref_out)
    assert (ref_n > 1).any()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("B,T,V", [(6, 4, 4099), (40, 8, 41000), (3, 5, 152064)])
def test_rows_behind_the_used_ones(kind, B, T, V):
    """The used rows as in a call of their own; the others masked, with nothing reported, whatever they and their parameters are."""
    M = B * T
    t, _ = batch(M, V, kind, 7, patterns=("bulk", "peaks", "flat"))
    n_used = np.resize([0, 1, T - 1, T, -3, T + 5], B).astype(np.int32)
    used = (np.arange(T)[None] < n_used[:, None]).reshape(-1)
    params = parameters(M, V, 7, "kpm")
    u = np.random.default_rng(3).random((M, 2)).astype(np.float32)
    want, rows = sample(t, params, u), filtered(t, params)
    assert want[4] == 0 and rows[3] == 0
    out_of = torch.from_numpy(~used).cuda()
    t[out_of, 1] = float("inf")
    params = [np.array(a) for a in params]
    params[0][~used] = np.resize(np.array([0.0, np.nan, -1.0], dtype=np.float32), M)[~used]
    u = u.copy()
    u[~used] = np.nan
    how = sd.Sampling(*params)
    n_dev = to_device(n_used)
    how.c.n_used, how.c.per = n_dev.data_ptr(), T
    tokens, prob, dense, lse, st = sample(t, None, u, how=how)
    assert st == 0
    for got, ref in zip((tokens, prob, dense, lse), want):
        np.testing.assert_array_equal(got[used], ref[used])
    assert (tokens[~used] == -1).all() and (prob[~used] == 0).all() and (dense[~used] == 0).all() and np.isneginf(lse[~used]).all()
    out, flse, kept = torch.full((M, V), 7.0, device="cuda"), torch.full((M,), 7.0, device="cuda"), torch.full((M,), -7, dtype=torch.int32, device="cuda")
    st = sd.new_status()
    sd.sd_filter_logits(t, how, out, flse, kept, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for got, ref in zip((out, flse, kept), rows):
        got = got.cpu().numpy()
        np.testing.assert_array_equal(got[used], ref[used])
        assert (np.isneginf(got[~used]) | (got[~used] == 0)).all()
