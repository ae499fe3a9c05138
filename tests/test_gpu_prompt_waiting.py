"""GPU: sequences that the pool of blocks does not suffice for take no part in a verify step: nothing of theirs, and nothing of the others', is
written; and the acceptance calls on trees that are marked so."""
import numpy as np
import pytest
import torch

from paper_2509_18824_b200 import binding as sd
from paper_2509_18824_b200 import workloads as wl
from paper_2509_18824_b200.step import VerifyStep, to_device

pytestmark = pytest.mark.gpu
bf = torch.bfloat16
T, V = 8, 1024


def workload(B, **over):
    a = dict(B=B, L=2, V=V, Hd=128, prefix=200, T=T)
    a.update(over)
    w = wl.make("c5", **a)
    w.parents = np.tile(wl.chain_tree(T)[None].astype(np.int32), (B, 1))
    w.n_nodes = np.full(B, T, dtype=np.int32)
    return w


def agreeable(vs):
    """Draft tokens that the target agrees with: a chain is accepted whole."""
    vs.lmhead()
    tok = torch.zeros_like(vs.draft_tok)
    tok[:, 1:] = vs.argmax.view(vs.w.B, T)[:, :-1]
    vs.draft_tok.copy_(tok)
    return tok


def fill(vs, p, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    N = p.prompts.N
    p.begin()
    for l in range(vs.L):
        qkv = torch.randn((N, 36, 128), generator=g, device="cuda").to(bf)
        out = torch.zeros((N, 28, 128), dtype=bf, device="cuda")
        p.layer(l, qkv[:, :28], qkv[:, 28:32], qkv[:, 32:], out)
    p.end()


def tails(vs):
    B = vs.w.B
    u, half = torch.zeros((B, T), device="cuda"), torch.full((B,), 0.5, device="cuda")
    q_rows = torch.full((B, T, V), 1.0 / V, device="cuda")
    how = sd.Sampling(inv_temp=np.ones(B * T, np.float32))
    return {"fused": vs.tail, "apart": lambda: (vs.lmhead(), vs.accept(), vs.compact()), "sampled": lambda: vs.tail_sampled(1.0, u, half),
            "sampled_apart": lambda: vs.tail_sampled(1.0, u, half, fused=False), "filtered": lambda: vs.tail_filtered(how, q_rows, u, half)}


def short_of_blocks(vs):
    """Three blocks: sequence 0 has 60 tokens and gave the block of its tree back, sequence 1 has taken it for its prompt."""
    p, held, given_back = take_all_blocks(vs)
    table = vs.batch.block_table.cpu().numpy()
    assert held.tolist() == [1, 2] and vs.batch.len.tolist() == [60, 100] and given_back in table[1, :2]
    vs.check_status()
    return p, held


def take_all_blocks(vs):
    pool, held = sd.BlockPool(3), torch.zeros(2, dtype=torch.int32, device="cuda")
    vs.batch.len.zero_()
    p = vs.prompts(60, [60, 0], pool, held)
    fill(vs, p, 1)
    p.reserve_trees()
    assert held.tolist() == [2, 1]
    given_back = int(vs.batch.block_table[0, 1])
    p = vs.prompts(100, [0, 100], pool, held)
    fill(vs, p, 2)
    return p, held, given_back


def expected(vs, before, who, at):
    """The caches behind a step that accepted all nodes of sequence `who`, at tokens `at` and on."""
    row = vs.batch.block_table.cpu().numpy()[who]
    want = [c.clone() for c in before]
    for c, tree in zip(want, vs.k_tree + vs.v_tree):
        for i in range(T):
            c[int(row[(at + i) // 64]), :, (at + i) % 64] = tree[who, i]
    return want


def same(got, want):
    return all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(got, want))


@pytest.mark.parametrize("tail", ["fused", "apart", "sampled", "sampled_apart", "filtered"])
def test_a_sequence_without_blocks_for_its_tree_waits(tail):
    vs = VerifyStep(workload(2))
    agreeable(vs)
    p, held = short_of_blocks(vs)
    before = [c.clone() for c in vs.k_cache + vs.v_cache]
    p.reserve_trees()
    for x in (vs.n_acc, vs.path, vs.out_tok, vs.new_len):
        x.fill_(77)
    vs.attention_layers()
    tails(vs)[tail]()
    torch.cuda.synchronize()
    vs.check_status()
    assert vs.n_acc.tolist() == [0, T] and vs.new_len.tolist() == [60, 100 + T] and held.tolist() == [1, 2]
    assert (vs.path[0] == -1).all() and (vs.out_tok[0] == -1).all() and vs.path[1].tolist() == list(range(T)) and (vs.out_tok[1] >= 0).all()
    assert same(vs.k_cache + vs.v_cache, expected(vs, before, 1, 100))
    assert all((o[0] == 0).all() and (o[1] != 0).any() for o in vs.out)
    # the other one is done: its blocks come back, and the first one's tree, as it was, goes on
    vs.batch.len.copy_(vs.new_len)
    vs.batch.len[1] = 0
    vs.batch.n_nodes[1] = 0
    before = [c.clone() for c in vs.k_cache + vs.v_cache]
    p.reserve_trees()
    vs.attention_layers()
    tails(vs)[tail]()
    torch.cuda.synchronize()
    vs.check_status()
    assert vs.n_acc.tolist() == [T, 0] and vs.new_len.tolist() == [60 + T, 0] and held.tolist() == [2, 0]
    assert same(vs.k_cache + vs.v_cache, expected(vs, before, 0, 60))


def test_a_captured_step_lets_sequences_wait_and_go_on():
    vs = VerifyStep(workload(2))
    agreeable(vs)
    p, held = short_of_blocks(vs)
    before = [c.clone() for c in vs.k_cache + vs.v_cache]
    p.reserve_trees()
    vs.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.reserve_trees()
        vs.run()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    vs.check_status()
    assert vs.n_acc.tolist() == [0, T] and same(vs.k_cache + vs.v_cache, expected(vs, before, 1, 100))
    vs.batch.len[1] = 0
    vs.batch.n_nodes[1] = 0
    before = [c.clone() for c in vs.k_cache + vs.v_cache]
    graph.replay()
    torch.cuda.synchronize()
    vs.check_status()
    assert vs.n_acc.tolist() == [T, 0] and held.tolist() == [2, 0] and same(vs.k_cache + vs.v_cache, expected(vs, before, 0, 60))


@pytest.mark.parametrize("call", ["fused", "apart", "sampled", "sampled_apart", "filtered", "chain", "chain_logits"])
def test_trees_that_take_no_part(call):
    B = 4
    vs, all_in = (VerifyStep(workload(B, prefix=100)) for _ in range(2))
    u, half = torch.zeros((B, T), device="cuda"), torch.full((B,), 0.5, device="cuda")
    for s in (vs, all_in):
        agreeable(s)
    vs.batch.n_nodes.copy_(to_device(np.array([T, -5, 0, -T], dtype=np.int32)))
    sd.sd_tree_prepare(vs.batch, vs.status)
    before = [c.clone() for c in vs.k_cache + vs.v_cache]
    for s in (vs, all_in):
        for x in (s.n_acc, s.path, s.out_tok, s.new_len):
            x.fill_(77)
        s.attention_layers()
        if call.startswith("chain"):
            M = B * T
            lse, logits = torch.zeros(M, device="cuda"), torch.zeros((M, V), device="cuda")
            need = sd.sd_workspace_bytes(s.batch, M, V)
            work = torch.empty(need, dtype=torch.uint8, device="cuda")
            sd.sd_lmhead_stats_logits(s.hidden, s.W, 1.0, None, None, lse, logits, work, s.status)
            q = torch.full((B, T, V), 1.0 / V, device="cuda")
            sd.sd_accept_chain_sampled(s.batch, s.hidden, s.W, 1.0, lse, s.draft_tok, q[:, :, 0].contiguous(), q, u, half, s.n_acc, s.path, s.out_tok, s.new_len,
                                       work, s.status, logits=logits if call == "chain_logits" else None)
            s.compact()
        else:
            tails(s)[call]()
    torch.cuda.synchronize()
    vs.check_status()
    all_in.check_status()
    for got, want in zip((vs.n_acc, vs.path, vs.out_tok, vs.new_len), (all_in.n_acc, all_in.path, all_in.out_tok, all_in.new_len)):
        assert torch.equal(got[0], want[0])
    assert vs.n_acc.tolist() == [T, 0, 0, 0] and vs.new_len[1:].tolist() == vs.batch.len[1:].tolist()
    assert (vs.path[1:] == -1).all() and (vs.out_tok[1:] == -1).all()
    assert same(vs.k_cache + vs.v_cache, expected(vs, before, 0, int(vs.w.len[0])))
    for o, l, full in zip(vs.out, vs.lse, all_in.out):
        assert torch.equal(o[0], full[0]) and (o[1:] == 0).all() and (l[1:] == 0).all()


@pytest.mark.parametrize("n", [-T - 1, T + 1])
def test_node_counts_out_of_range_are_still_reported(n):
    for call in ("fused", "apart", "sampled", "filtered"):
        vs = VerifyStep(workload(1))
        vs.batch.n_nodes.fill_(n)
        tails(vs)[call]()
        torch.cuda.synchronize()
        assert int(vs.status.item()) == sd.SD_ERR_INVALID_TREE
    vs.status.zero_()
    sd.sd_tree_prepare(vs.batch, vs.status)
    torch.cuda.synchronize()
    assert int(vs.status.item()) == sd.SD_ERR_INVALID_TREE


def test_masks_of_a_tree_that_waits_are_made():
    vs = VerifyStep(workload(2))
    want = vs.batch.anc_mask.clone()
    vs.batch.anc_mask.fill_(-1)
    vs.batch.n_nodes.neg_()
    sd.sd_tree_prepare(vs.batch, vs.status)
    torch.cuda.synchronize()
    vs.check_status()
    assert torch.equal(vs.batch.anc_mask, want)


@pytest.mark.parametrize("tail", ["fused", "sampled", "filtered"])
def test_a_step_whose_trees_have_no_blocks_is_reported(tail):
    """Blocks for the trees have not been reserved: nothing goes to blocks that were given back."""
    vs = VerifyStep(workload(2))
    agreeable(vs)
    _, held = short_of_blocks(vs)
    before = [c.clone() for c in vs.k_cache + vs.v_cache]
    vs.attention_layers()
    tails(vs)[tail]()
    torch.cuda.synchronize()
    assert int(vs.status.item()) == sd.SD_ERR_BOUNDS
    # what fits into the blocks that they hold is there, and nothing else
    row, want = vs.batch.block_table.cpu().numpy(), [c.clone() for c in before]
    for c, tree in zip(want, vs.k_tree + vs.v_tree):
        for b, at in ((0, 60), (1, 100)):
            for i in range(T):
                if at + i < 64 * int(held[b]):
                    c[int(row[b, (at + i) // 64]), :, (at + i) % 64] = tree[b, i]
    assert same(vs.k_cache + vs.v_cache, want)


def test_table_entries_behind_a_sequences_blocks_name_none():
    vs = VerifyStep(workload(2))
    vs.batch.block_table.fill_(5)
    p, held = short_of_blocks(vs)
    p.reserve_trees()
    torch.cuda.synchronize()
    vs.check_status()
    table = vs.batch.block_table.cpu().numpy()
    for b in range(2):
        assert (table[b, :int(held[b])] >= 0).all() and (table[b, int(held[b]):] == -1).all()
