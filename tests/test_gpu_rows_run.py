"""GPU: the operators on rows of logits together, as they are used: drafts sampled from a draft model's rows and verified against the
filtered target; a draft that learns from its target's first logits."""
import numpy as np
import pytest
import torch

import oracle
from oracle import rows as ref
from oracle import sampling as smp
from paper_2509_18824_b200 import binding as sd
from paper_2509_18824_b200 import workloads as wl
from paper_2509_18824_b200.step import VerifyStep, to_device
from test_gpu_sampled import decisive_chain_inputs, decisive_tree_inputs

pytestmark = pytest.mark.gpu


def target_rows(vs, params):
    """The filtered target of every row, in 64 bits, from the logits that the LM head leaves (before the call that filters them)."""
    M, V = vs.w.B * vs.w.T_max, vs.w.V
    lse, logits = torch.zeros(M, device="cuda"), torch.zeros((M, V), device="cuda")
    sd.sd_lmhead_stats_logits(vs.hidden, vs.W, 1.0, None, None, lse, logits, vs.workspace, vs.status)
    torch.cuda.synchronize()
    x = logits.double().cpu().numpy()
    it, k, p, mp = params
    return np.stack([ref.probabilities(x[r], inv_temp=float(it[r]), top_k=int(k[r]), top_p=float(p[r]), min_p=float(mp[r])) for r in range(M)]), x


def drafts(w, x, seed, N, kind):
    """A draft model's rows (the target's and noise), tokens drawn from them at a temperature behind top-k: (rows' distributions, tokens
    and probabilities of N draws per row)."""
    g = np.random.default_rng(seed)
    M, V = x.shape
    rows = torch.from_numpy((x + g.standard_normal(x.shape) * 0.4).astype(np.float32)).cuda().to(torch.bfloat16 if kind == "bf16" else torch.float32)
    how = sd.Sampling(np.full(M, 0.9, np.float32), np.resize([0, 40], M).astype(np.int32), np.full(M, 0.98, np.float32))
    u = torch.from_numpy(g.random((M, N)).astype(np.float32)).cuda()
    tokens, prob, probs, st = torch.zeros((M, N), dtype=torch.int32, device="cuda"), torch.zeros((M, N), device="cuda"), torch.zeros((M, V), device="cuda"), sd.new_status()
    sd.sd_sample_logits(rows, how, u, tokens, prob, probs, None, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    return probs, tokens.cpu().numpy(), prob.cpu().numpy()


def target_parameters(M):
    return (np.resize([0.8, 1.0, 1.3], M).astype(np.float32), np.resize([0, 100, 0, 20], M).astype(np.int32),
            np.resize([0.95, 1.0, 0.9], M).astype(np.float32), np.resize([0.0, 0.02], M).astype(np.float32))


def log_rows(p):
    with np.errstate(divide="ignore"):
        return np.log(p)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("cfg,over", [("c1", dict()), ("c5", dict(B=3, L=2, V=8192, Hd=128, prefix=100)), ("c4", dict(L=1, V=4099, Hd=256, prefix_range=(40, 300)))])
def test_sampled_trees_against_the_filtered_target(cfg, over, kind):
    w = wl.make(cfg, hidden_gain=12.0, **over)
    B, T = w.B, w.T_max
    M = B * T
    vs = VerifyStep(w)
    params = target_parameters(M)
    p64, x = target_rows(vs, params)
    most = max(int(np.bincount(w.parents[b][1:int(w.n_nodes[b])], minlength=1).max()) if int(w.n_nodes[b]) > 1 else 1 for b in range(B))
    probs, tokens, _ = drafts(w, x, 5, most, kind)
    tok = np.zeros((B, T), dtype=np.int32)
    for b in range(B):
        seen = np.zeros(T, dtype=int)
        for j in range(1, int(w.n_nodes[b])):
            i = int(w.parents[b][j])
            tok[b, j] = tokens[b * T + i, seen[i]]
            seen[i] += 1
    vs.draft_tok.copy_(to_device(tok))
    q_rows = probs.view(B, T, -1)
    q = q_rows.cpu().numpy()
    g = np.random.default_rng(6)
    moved = 0
    for _ in range(3 if B > 1 else 8):
        u, wv, ref_n, ref_path, ref_out, _ = decisive_tree_inputs(w, tok, q, log_rows(p64), 1.0, g)
        vs.tail_filtered(sd.Sampling(*params), q_rows, to_device(u), to_device(wv))
        torch.cuda.synchronize()
        vs.check_status()
        np.testing.assert_array_equal(vs.n_acc.cpu().numpy(), ref_n)
        np.testing.assert_array_equal(vs.path.cpu().numpy(), ref_path)
        np.testing.assert_array_equal(vs.out_tok.cpu().numpy(), ref_out)
        np.testing.assert_array_equal(vs.new_len.cpu().numpy(), w.len + ref_n)
        for b in range(B):                                    # nothing is emitted that the filters took out
            at = [0] + [int(n) for n in ref_path[b][1:ref_n[b]]]
            assert all(p64[b * T + i, t] > 0 for i, t in zip(at, ref_out[b]))
        moved += int((ref_n > 1).sum())
    assert moved > 0
    # the KV of the survivors joined the cache as in a step of its own
    alone = VerifyStep(w)
    alone.n_acc.copy_(vs.n_acc)
    alone.path.copy_(vs.path)
    alone.compact()
    again = VerifyStep(w)
    again.draft_tok.copy_(vs.draft_tok)
    again.tail_filtered(sd.Sampling(*params), q_rows, to_device(u), to_device(wv))
    torch.cuda.synchronize()
    for a, b in zip(alone.k_cache + alone.v_cache, again.k_cache + again.v_cache):
        assert torch.equal(a, b)


def test_sampled_chains_against_the_filtered_target():
    w = wl.make("chain11", attention=False, hidden_gain=12.0, L=1, V=3000, Hd=128, prefix=70)
    wl.fill_attention(w, [0])
    B, T = w.B, w.T_max
    M, V = B * T, w.V
    vs = VerifyStep(w)
    params = target_parameters(M)
    p64, x = target_rows(vs, params)
    probs, tokens, prob = drafts(w, x, 7, 1, "f32")
    tok, q_tok = np.zeros((B, T), dtype=np.int32), np.zeros((B, T), dtype=np.float32)
    tok[:, 1:] = tokens.reshape(B, T)[:, :-1]
    q_tok[:, 1:] = prob.reshape(B, T)[:, :-1]
    q_rows = probs.view(B, T, V)
    g = np.random.default_rng(8)
    u, wv, ref_n, ref_out = decisive_chain_inputs(w, tok, q_rows.cpu().numpy(), lambda r: p64[r], g)
    lse, logits, flse = torch.zeros(M, device="cuda"), torch.zeros((M, V), device="cuda"), torch.zeros(M, device="cuda")
    sd.sd_lmhead_stats_logits(vs.hidden, vs.W, 1.0, None, None, lse, logits, vs.workspace, vs.status)
    sd.sd_filter_logits(logits, sd.Sampling(*params), logits, flse, None, vs.status)
    ws = torch.zeros(sd.sd_workspace_bytes(vs.batch, M, V), dtype=torch.uint8, device="cuda")
    sd.sd_accept_chain_sampled(vs.batch, vs.hidden, vs.W, 1.0, flse, to_device(tok), to_device(q_tok), q_rows, to_device(u), to_device(wv),
                               vs.n_acc, vs.path, vs.out_tok, vs.new_len, ws, vs.status, logits=logits)
    torch.cuda.synchronize()
    vs.check_status()
    np.testing.assert_array_equal(vs.n_acc.cpu().numpy(), ref_n)
    np.testing.assert_array_equal(vs.out_tok.cpu().numpy(), ref_out)


def test_a_step_of_the_drafts_training():
    """Target rows from its hidden states, their first entries and arg-max, the draft's loss and the gradient of its head's weights,
    against the formulas in 64 bits on the same rows."""
    M, Hd, V, K = 96, 128, 4099, 32
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    Wt = (torch.randn((V, Hd), generator=g, device="cuda") * 0.2).bfloat16()
    ht = torch.randn((M, Hd), generator=g, device="cuda").bfloat16()
    hs = (ht.float() + 0.5 * torch.randn((M, Hd), generator=g, device="cuda")).bfloat16()
    Ws = (Wt.float() + 0.05 * torch.randn((V, Hd), generator=g, device="cuda")).requires_grad_()
    f, i = (lambda *s: torch.zeros(s, device="cuda")), (lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda"))
    logits, lse, st = f(M, V), f(M), sd.new_status()
    ws = torch.zeros(sd.sd_workspace_bytes(None, M, V), dtype=torch.uint8, device="cuda")
    sd.sd_lmhead_stats_logits(ht, Wt, 1.0, None, None, lse, logits, ws, st)
    val, idx, top_lse, kl, ce = f(M, K), i(M, K), f(M), f(M), f(M)
    sd.sd_top_logits(logits, 1.0, val, idx, top_lse, st)
    student = hs.float() @ Ws.t()
    weight = torch.full((M,), 1.0 / M, device="cuda")
    grad = torch.zeros_like(student)
    sd.sd_distill_loss(student.detach(), val, idx, top_lse, idx[:, 0].contiguous(), 1.0, 1.0, 0.1, kl, ce, None, weight, grad, st)
    student.backward(grad)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    z, t = student.detach().double().cpu().numpy(), logits.double().cpu().numpy()
    want, off = np.zeros((M, V)), np.zeros((M, V))
    for r in range(M):
        v, at, l = ref.top(t[r], K, 1.0)
        np.testing.assert_array_equal(idx[r].cpu().numpy(), at)
        # (the target's log-sum-exp is handed on in 32 bits)
        a, b, want[r] = ref.distill(z[r], v, at, float(top_lse[r]), int(at[0]), 1.0, 1.0, 0.1, 1.0 / M)
        assert abs(float(kl[r]) - a) <= 2e-6 + 2.0 ** -23 * abs(a) and abs(float(ce[r]) - b) <= 2e-6 + 2.0 ** -23 * abs(b)
        # an entry of the gradient: 8e-6 of the student's share (and as much for the rest's ratio), 4e-6 of the target's, a rounding
        s = np.exp(z[r] - ref.lse(z[r]))
        off[r] = 2.0 ** -24 * np.abs(want[r]) + 1.1 / M * 16e-6 * s
        off[r, at] += 1.1 / M * 4e-6 * np.minimum(1.0, np.exp(v - float(top_lse[r])))
        off[r, at[0]] += 1.1 / M * 3 * 2.0 ** -24
    # the product: those, and at most M roundings of the sum of M terms
    want, off, h = torch.from_numpy(want).cuda(), torch.from_numpy(off).cuda(), hs.double()
    bound = off.t() @ h.abs() + M * 2.0 ** -24 * ((want.abs() + off).t() @ h.abs())
    assert ((Ws.grad.double() - want.t() @ h).abs() <= bound).all()
