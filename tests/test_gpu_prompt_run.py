"""GPU: the calls on packed new tokens together, as they are used: prompts in pieces into the empty caches of a verify step, its trees over
them, acceptance and compaction, and tables that follow."""
import numpy as np
import pytest
import torch

import oracle
from oracle import prompt as ref
from paper_2509_18824_b200 import binding as sd
from paper_2509_18824_b200 import workloads as wl
from paper_2509_18824_b200.step import VerifyStep, to_device
from gpu_util import check_attention
from prompt_util import blocks

pytestmark = pytest.mark.gpu


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("heads", [(28, 4), (4, 4), (7, 1)], ids=str)
def test_prompts_then_trees(heads):
    Hq, Hkv = heads
    prompt = np.array([150, 1, 333, 64, 19], dtype=np.int32)
    B, L, T = 5, 2, 12
    w = wl.make("c5", B=B, L=L, Hq=Hq, Hkv=Hkv, V=1024, Hd=128, prefix=int(prompt.max()), T=T)
    vs = VerifyStep(w)
    batch = vs.batch
    # nothing is cached, nobody holds a block, and what the caches hold is not a number
    batch.len.zero_()
    num_blocks = int(vs.k_cache[0].shape[0])
    batch.block_table.fill_(2 ** 30)
    for c in vs.k_cache + vs.v_cache:
        c.fill_(0x7fc0)
    pool = sd.BlockPool(num_blocks)
    held = torch.zeros(B, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    ks, vs_ = ([torch.zeros((B, int(prompt.max()), Hkv, 128), dtype=torch.bfloat16, device="cuda") for _ in range(L)] for _ in range(2))
    bf = torch.bfloat16
    done = np.zeros(B, dtype=np.int32)
    for piece in ([100, 1, 64, 0, 18], [50, 0, 200, 64, 1], [0, 0, 69, 0, 0]):
        new = np.array(piece, dtype=np.int32)
        N = int(new.sum()) + 2
        start = np.concatenate([[0], np.cumsum(new)])
        p = vs.prompts(N, new, pool, held)
        p.begin()
        for l in range(L):
            qkv = torch.randn((N, Hq + 2 * Hkv, 128), generator=g, device="cuda").to(bf)
            out, lse = torch.zeros((N, Hq, 128), dtype=bf, device="cuda"), torch.zeros((N, Hq), device="cuda")
            q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
            p.layer(l, q, k, v, out, lse)
            torch.cuda.synchronize()
            vs.check_status()
            kc, vc = f64(vs.k_cache[l].view(bf)), f64(vs.v_cache[l].view(bf))
            want, want_lse, spread, size = ref.attention(f64(q)[:N - 2], kc, vc, f64(batch.block_table).astype(np.int64), done, new, vs.scale)
            bound = (2.0 ** -8 + 2.0 ** -10) * spread + 2.0 ** -8 * np.abs(want)
            assert (np.abs(f64(out)[:N - 2] - want) <= bound).all()
            assert (np.abs(f64(lse)[:N - 2] - want_lse) <= 2.0 ** -24 * (128 * size + 500) + 2.0 ** -22 * np.abs(want_lse)).all()
            for b in range(B):
                n, c = int(new[b]), int(done[b])
                ks[l][b, c:c + n], vs_[l][b, c:c + n] = k[start[b]:start[b] + n], v[start[b]:start[b] + n]
        p.end()
        done += new
        np.testing.assert_array_equal(batch.len.cpu().numpy(), done)
        np.testing.assert_array_equal(held.cpu().numpy(), [blocks(int(d)) for d in done])
    np.testing.assert_array_equal(done, prompt)
    # the trees of the step, over what the prompts left
    p.reserve_trees()
    vs.run()
    torch.cuda.synchronize()
    vs.check_status()
    np.testing.assert_array_equal(held.cpu().numpy(), [blocks(int(d) + int(n)) for d, n in zip(prompt, w.n_nodes)])
    table = batch.block_table.cpu().numpy()
    owned = np.concatenate([table[b, :int(held[b])] for b in range(B)])
    assert np.unique(owned).size == owned.size and owned.min() >= 0 and owned.max() < num_blocks
    G = oracle.Geometry.of(type("W", (), dict(B=B, T_max=w.T_max, Hq=Hq, Hkv=Hkv, D=128, block_table=np.where((table >= 0) & (table < num_blocks), table, 0).astype(np.int32),
                                              len=prompt, n_nodes=w.n_nodes, parents=w.parents)))
    for l in range(L):
        before = [np.zeros((num_blocks, Hkv, 64, 128), dtype=np.uint16) for _ in range(2)]
        for cache, rows in zip(before, (ks[l], vs_[l])):
            x = rows.view(torch.int16).cpu().numpy().view(np.uint16)
            for b in range(B):
                for t in range(int(prompt[b])):
                    cache[table[b, t // 64], :, t % 64] = x[b, t]
        want, _ = oracle.attention(G, before[0], before[1], w.q[l], w.k_tree[l], w.v_tree[l], w.scale)
        check_attention(vs.out[l].float().cpu().numpy(), want, f"layer {l}")
        # the accepted nodes behind the prompts, and what was there before
        n_acc, path = vs.n_acc.cpu().numpy(), vs.path.cpu().numpy()
        for cache, tree, now in zip(before, (w.k_tree[l], w.v_tree[l]), (vs.k_cache[l], vs.v_cache[l])):
            got = now.cpu().numpy().view(np.uint16)
            for b in range(B):
                for i in range(int(n_acc[b])):
                    t = int(prompt[b]) + i
                    cache[table[b, t // 64], :, t % 64] = tree[b, path[b, i]]
                for t in range(int(prompt[b]) + int(n_acc[b])):
                    assert np.array_equal(got[table[b, t // 64], :, t % 64], cache[table[b, t // 64], :, t % 64])
    # behind acceptance: the next step's tables, from lengths that only the device knows; then everything comes back
    batch.len.copy_(vs.new_len)
    p.reserve_trees()
    torch.cuda.synchronize()
    np.testing.assert_array_equal(held.cpu().numpy(), [blocks(int(d) + int(a) + int(n)) for d, a, n in zip(prompt, vs.n_acc.tolist(), w.n_nodes)])
    nothing = torch.zeros(B, dtype=torch.int32, device="cuda")
    sd.sd_assign_blocks(pool, batch.block_table, held, nothing, nothing, None, vs.status)
    torch.cuda.synchronize()
    vs.check_status()
    assert int(pool.n_free.item()) == num_blocks and sorted(pool.free_blocks.tolist()) == list(range(num_blocks))


def test_sequences_that_the_pool_does_not_suffice_for_wait():
    w = wl.make("c5", B=3, L=1, V=1024, Hd=128, prefix=200, T=8)
    vs = VerifyStep(w)
    vs.batch.len.zero_()
    pool = sd.BlockPool(3)                                   # of 2, 2 and 1 that are needed
    held = torch.zeros(3, dtype=torch.int32, device="cuda")
    new = np.array([100, 100, 30], dtype=np.int32)
    p = vs.prompts(230, new, pool, held)
    p.begin()
    qkv = torch.randn((230, 36, 128), device="cuda").to(torch.bfloat16)
    out = torch.full((230, 28, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    p.layer(0, qkv[:, :28], qkv[:, 28:32], qkv[:, 32:], out)
    p.end()
    torch.cuda.synchronize()
    vs.check_status()
    assert p.granted.tolist() == [1, 0, 0] and vs.batch.len.tolist() == [100, 0, 0] and held.tolist() == [2, 0, 0]
    assert (out[100:] == 5.0).all() and not (out[:100] == 5.0).all(dim=2).any()
    with pytest.raises(AssertionError):
        vs.prompts(230, new, pool)


def test_a_step_on_another_stream():
    w = wl.make("c5", B=2, L=1, V=1024, Hd=128, prefix=200, T=8)
    vs = VerifyStep(w)
    vs.batch.len.zero_()
    pool = sd.BlockPool(int(vs.k_cache[0].shape[0]))
    held = torch.zeros(2, dtype=torch.int32, device="cuda")
    p = vs.prompts(90, [60, 30], pool, held)
    qkv = torch.randn((90, 36, 128), device="cuda").to(torch.bfloat16)
    out, here = (torch.zeros((90, 28, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    p.begin(s)
    p.layer(0, qkv[:, :28], qkv[:, 28:32], qkv[:, 32:], out, stream=s)
    p.end(s)
    s.synchronize()
    vs.check_status()
    assert vs.batch.len.tolist() == [60, 30]
    vs.batch.len.zero_()
    p.begin()
    p.layer(0, qkv[:, :28], qkv[:, 28:32], qkv[:, 32:], here)
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), here.view(torch.int16)) and out.any()


def test_without_a_pool_the_tables_are_the_callers():
    w = wl.make("c5", B=2, L=1, V=1024, Hd=128, prefix=200, T=8)
    vs = VerifyStep(w)
    vs.batch.len.zero_()
    before = vs.batch.block_table.clone()
    p = vs.prompts(90, [60, 30])
    qkv = torch.randn((90, 36, 128), device="cuda").to(torch.bfloat16)
    out = torch.zeros((90, 28, 128), dtype=torch.bfloat16, device="cuda")
    p.begin()
    p.layer(0, qkv[:, :28], qkv[:, 28:32], qkv[:, 32:], out)
    p.end()
    torch.cuda.synchronize()
    vs.check_status()
    assert vs.batch.len.tolist() == [60, 30] and torch.equal(before, vs.batch.block_table) and out.any(dim=2).all()
    with pytest.raises(AssertionError):
        p.reserve_trees()
