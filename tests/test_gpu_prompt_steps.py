"""GPU: prompts brought into a verify step's caches in the ways that a serving program calls them: input sets that alternate, streams that
are not the constructor's, objects dropped early, pieces that do not fit."""
import numpy as np
import pytest
import torch

from paper_2509_18824_b200 import binding as sd
from paper_2509_18824_b200.step import VerifyStep
from test_gpu_prompt_waiting import T, agreeable, bf, expected, fill, same, short_of_blocks, workload

pytestmark = pytest.mark.gpu


def host_step(B, **over):
    vs = VerifyStep(workload(B, **over), keep_host_inputs=True)
    tok = agreeable(vs)
    vs.host["draft_tok"].copy_(tok)
    torch.cuda.synchronize()
    return vs


def test_prompts_and_steps_from_the_host():
    """The step's inputs exist twice; its tables and lengths once."""
    vs = host_step(2)
    pool, held = sd.BlockPool(8), torch.zeros(2, dtype=torch.int32, device="cuda")
    vs.batch.len.zero_()
    p = vs.prompts(173, [130, 43], pool, held)
    fill(vs, p, 3)
    lens = [130, 43]
    for step in range(4):
        torch.cuda.synchronize()
        before = [c.clone() for c in vs.k_cache + vs.v_cache]
        if step == 3:                                        # another piece in between
            more = vs.prompts(30, [0, 30], pool, held)
            fill(vs, more, 4)
            lens[1] += 30
            torch.cuda.synchronize()
            before = [c.clone() for c in vs.k_cache + vs.v_cache]
        vs.run_from_host()
        torch.cuda.synchronize()
        vs.check_status()
        assert vs.host_out["n_acc"].tolist() == [T, T] and vs.host_out["new_len"].tolist() == [n + T for n in lens], step
        assert held.tolist() == [-(-(n + T) // 64) for n in lens]
        want = expected(vs, expected(vs, before, 0, lens[0]), 1, lens[1])
        assert same(vs.k_cache + vs.v_cache, want), step
        vs.batch.len.copy_(vs.new_len)
        lens = [n + T for n in lens]
    table = vs.batch.block_table.cpu().numpy()
    owned = np.concatenate([table[b, :int(held[b])] for b in range(2)])
    assert np.unique(owned).size == owned.size


def test_steps_from_the_host_let_sequences_wait():
    vs = host_step(2)
    p, held = short_of_blocks(vs)
    for _ in range(3):
        torch.cuda.synchronize()
        at = int(vs.batch.len[1])
        before = [c.clone() for c in vs.k_cache + vs.v_cache]
        vs.run_from_host()
        torch.cuda.synchronize()
        vs.check_status()
        assert vs.host_out["n_acc"].tolist() == [0, T] and vs.host_out["new_len"].tolist() == [60, at + T]
        assert same(vs.k_cache + vs.v_cache, expected(vs, before, 1, at))
        vs.batch.len.copy_(vs.new_len)
    assert held.tolist() == [1, 2]


def test_tables_and_lengths_exist_once():
    vs = host_step(2)
    a, b = (s["batch"] for s in vs._slots)
    assert a.len is b.len and a.block_table.data_ptr() == b.block_table.data_ptr() and a.c.len == b.c.len and a.c.block_table == b.c.block_table
    assert a.n_nodes.data_ptr() != b.n_nodes.data_ptr() and a.parents.data_ptr() != b.parents.data_ptr() and a.anc_mask.data_ptr() != b.anc_mask.data_ptr()


def test_without_prompts_steps_from_the_host_keep_their_lengths():
    vs = host_step(2)
    for _ in range(3):
        vs.run_from_host()
    torch.cuda.synchronize()
    vs.check_status()
    assert vs.host_out["new_len"].tolist() == [int(n) + T for n in vs.w.len]


@pytest.mark.parametrize("given", ["int32", "int64"])
def test_a_step_made_while_its_stream_is_busy(given):
    """Everything that the object makes is ready on the stream of its calls."""
    w = workload(3, L=1)
    vs = VerifyStep(w)
    pool, held = sd.BlockPool(3), torch.zeros(3, dtype=torch.int32, device="cuda")       # of 2, 2 and 1 blocks that are needed
    new = torch.tensor([100, 100, 30], dtype=getattr(torch, given), device="cuda")
    qkv = torch.randn((230, 36, 128), device="cuda").to(bf)
    out = torch.full((230, 28, 128), 5.0, dtype=bf, device="cuda")
    vs.batch.len.zero_()
    vs.prompts(230, new, pool, held).begin()                 # (loads the kernels; takes blocks that the next begin finds held)
    torch.cuda.synchronize()
    assert held.tolist() == [2, 0, 0]
    side = torch.cuda.Stream()
    for _ in range(3):
        vs.batch.len.zero_()
        out.fill_(5.0)
        torch.cuda.synchronize()
        torch.cuda._sleep(50000000)                          # the current stream is busy for some 25 milliseconds
        p = vs.prompts(230, new, pool, held)
        p.begin(side)
        p.layer(0, qkv[:, :28], qkv[:, 28:32], qkv[:, 32:], out, stream=side)
        p.end(side)
        torch.cuda.synchronize()
        vs.check_status()
        assert p.granted.tolist() == [1, 0, 0] and vs.batch.len.tolist() == [100, 0, 0] and held.tolist() == [2, 0, 0]
        assert (out[100:] == 5.0).all() and not (out[:100] == 5.0).all(dim=2).any()


def test_memory_of_a_step_that_is_dropped_is_not_given_away_while_it_runs():
    w = workload(2, L=1)
    vs = VerifyStep(w)
    vs.batch.len.zero_()
    pool, held = sd.BlockPool(8), torch.zeros(2, dtype=torch.int32, device="cuda")
    qkv = torch.randn((90, 36, 128), device="cuda").to(bf)
    out = torch.zeros((90, 28, 128), dtype=bf, device="cuda")
    new = torch.tensor([60, 30], dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    p = vs.prompts(90, new, pool, held)
    for _ in range(2):                                       # (the first time loads the kernels, which takes as long as the pause below)
        p.begin(side)
        p.layer(0, qkv[:, :28], qkv[:, 28:32], qkv[:, 32:], out, stream=side)
        p.end(side)
    torch.cuda.synchronize()
    vs.batch.len.zero_()
    torch.cuda.synchronize()
    p = vs.prompts(90, new, pool, held)
    taken = {t.data_ptr(): t.numel() * t.element_size() for t in (p.workspace, p.granted)}
    sizes = list(taken.values())
    with torch.cuda.stream(side):
        torch.cuda._sleep(100000000)
    p.begin(side)
    p.layer(0, qkv[:, :28], qkv[:, 28:32], qkv[:, 32:], out, stream=side)
    p.end(side)
    del p
    got = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(6)]
    assert not side.query()                                  # (it still runs)
    assert not any(t.data_ptr() in taken for t in got)
    torch.cuda.synchronize()
    vs.check_status()
    assert vs.batch.len.tolist() == [60, 30]


def pieces(vs, p, N):
    qkv = torch.randn((N, 36, 128), device="cuda").to(bf)
    out = torch.zeros((N, 28, 128), dtype=bf, device="cuda")
    p.begin()
    for l in range(vs.L):
        p.layer(l, qkv[:, :28], qkv[:, 28:32], qkv[:, 32:], out)
    p.end()
    torch.cuda.synchronize()


@pytest.mark.parametrize("pooled", [True, False])
def test_tokens_that_had_no_rows_do_not_count_as_cached(pooled):
    vs = VerifyStep(workload(4, L=1))
    vs.batch.len.zero_()
    with_pool = (sd.BlockPool(int(vs.k_cache[0].shape[0])), torch.zeros(4, dtype=torch.int32, device="cuda")) if pooled else ()
    for N, want in ((120, [60, 60, 0, 0]), (130, [60, 60, 0, 0]), (119, [60, 0, 0, 0]), (0, [0, 0, 0, 0])):      # of 60, 60, 30 and 5
        vs.batch.len.zero_()
        vs.status.zero_()
        pieces(vs, vs.prompts(N, [60, 60, 30, 5], *with_pool), N)
        assert int(vs.status.item()) == sd.SD_ERR_BOUNDS
        assert vs.batch.len.tolist() == want, N


def test_tokens_that_the_table_has_no_room_for_do_not_count_as_cached():
    vs = VerifyStep(workload(3, L=1))
    room = 64 * vs.batch.max_blocks
    vs.batch.len.copy_(torch.tensor([10, 7, room - 20], dtype=torch.int32))
    pieces(vs, vs.prompts(room + 50, [room, 20, 21]), room + 50)
    assert int(vs.status.item()) == sd.SD_ERR_BOUNDS and vs.batch.len.tolist() == [10, 27, room - 20]
    vs.status.zero_()
    pieces(vs, vs.prompts(50, [-5, 20, 20]), 50)
    assert int(vs.status.item()) == sd.SD_ERR_INVALID_ARG and vs.batch.len.tolist() == [10, 47, room]


def test_blocks_for_trees_come_behind_the_prompts():
    vs = VerifyStep(workload(2, L=1))
    vs.batch.len.zero_()
    pool, held = sd.BlockPool(3), torch.zeros(2, dtype=torch.int32, device="cuda")
    p = vs.prompts(120, [60, 60], pool, held)
    p.begin()
    with pytest.raises(AssertionError):                      # (it would take the blocks of the new tokens back)
        p.reserve_trees()
    p.end()
    p.reserve_trees()
    torch.cuda.synchronize()
    vs.check_status()
    assert p.granted.tolist() == [1, 1] and p.trees_granted.tolist() == [1, 0] and held.tolist() == [2, 1] and vs.batch.len.tolist() == [60, 60]


def test_a_begin_that_failed_leaves_the_trees_their_blocks(monkeypatch):
    vs = VerifyStep(workload(2, L=1))
    vs.batch.len.zero_()
    pool, held = sd.BlockPool(8), torch.zeros(2, dtype=torch.int32, device="cuda")
    p = vs.prompts(120, [60, 60], pool, held)

    def refused(*_):
        raise sd.SdError(sd.SD_ERR_UNSUPPORTED)
    monkeypatch.setattr(sd, "sd_prompt_prepare", refused)
    with pytest.raises(sd.SdError):
        p.begin()
    monkeypatch.undo()
    p.reserve_trees()
    torch.cuda.synchronize()
    vs.check_status()
    assert held.tolist() == [1, 1] and p.trees_granted.tolist() == [1, 1] and vs.batch.len.tolist() == [0, 0]
