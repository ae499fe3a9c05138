"""GPU: causal attention of packed new tokens over the paged cache, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from paper_2509_18824_b200 import binding as sd
from prompt_util import Requests

pytestmark = pytest.mark.gpu

# (new, cached) of the requests of a call: single tokens, tiles' and blocks' edges (64 keys a block, 128 a tile, 18 or 128 tokens a row
# tile), whole prompts, chunks behind a prefix, requests without new tokens
BATCHES = {
    "one": [(1, 0)],
    "one_more": [(1, 64)],
    "singles": [(1, c) for c in (0, 1, 62, 63, 64, 65, 126, 127, 128, 129, 200, 511)],
    "block_edges": [(n, 0) for n in (1, 2, 63, 64, 65, 127, 128, 129)],
    "row_tiles": [(n, 5) for n in (17, 18, 19, 35, 36, 37, 16, 32, 33)],
    "prompt": [(700, 0)],
    "chunks": [(61, 1000), (1, 3000), (130, 77), (0, 100), (256, 256)],
    "with_idle": [(0, 0), (5, 3), (0, 64), (0, 0), (70, 0), (0, 1)],
    "long_single": [(1, 9000), (3, 20)],
}


@pytest.mark.parametrize("heads", [(4, 4), (7, 1), (28, 4), (8, 1), (6, 2), (5, 1), (3, 3)], ids=str)
@pytest.mark.parametrize("batch", BATCHES)
def test_against_the_oracle(batch, heads):
    r = Requests(BATCHES[batch], *heads, seed=len(batch) + heads[0])
    r.prepare()
    r.append()
    r.attend()
    r.check()


@pytest.mark.parametrize("seed", range(6))
def test_drawn_batches(seed):
    g = np.random.default_rng(100 + seed)
    lens = [(int(g.integers(0, g.choice([2, 40, 400]))), int(g.integers(0, g.choice([3, 200, 2500])))) for _ in range(int(g.integers(1, 24)))]
    lens.append((1, 0))
    Hkv = int(g.choice([1, 2, 4]))
    r = Requests(lens, Hkv * int(g.integers(1, 9)), Hkv, seed=seed, strided=bool(seed % 2))
    r.prepare()
    r.append()
    r.attend()
    r.check()


@pytest.mark.parametrize("gain", [0.0, 30.0, 200.0])
def test_flat_and_peaked_rows(gain):
    """Equal scores; scores in the hundreds, where one key has nearly all the weight and references move."""
    r = Requests([(150, 0), (1, 700), (40, 300)], 7, 1, seed=5, gain=gain)
    if gain == 0.0:
        r.q[:r.rows] = 0.0
    r.prepare()
    r.append()
    r.attend()
    torch.cuda.synchronize()
    out, lse, spread, size = r.expect()
    # (128 products of this size differ by up to 2^-17 of it in a score, and so the weights by as much)
    got = r.out[:r.rows].double().cpu().numpy()
    slack = 2.0 ** -17 * size[..., None] * 2.0
    bound = (2.0 ** -8 + 2.0 ** -10 + slack) * spread + (2.0 ** -8 + slack) * np.abs(out) + 1e-30
    assert (np.abs(got - out) <= bound).all()
    assert (np.abs(r.lse[:r.rows].double().cpu().numpy() - lse) <= 2.0 ** -17 * size + 2.0 ** -22 * np.abs(lse) + 2.0 ** -14).all()


def test_rising_scores():
    """Each block of keys towers over the one before: the row's reference is raised time and again."""
    r = Requests([(200, 600), (1, 800)], 4, 2, seed=8)
    r.prepare()
    r.append()
    r.q[:r.rows] = 1.0
    ramp = torch.arange(r.num_blocks * 64, device="cuda").float()
    for b, (n, c) in enumerate(r.lens):
        for t in range(n + c):
            r.k_cache[r.table[b, t // 64], :, t % 64] = 0.09 * float(ramp[t])           # scores up to 11.3 x 72: rises by 93 a block
    r.attend()
    torch.cuda.synchronize()
    out, lse, spread, size = r.expect()
    got = r.out[:r.rows].double().cpu().numpy()
    slack = 2.0 ** -17 * size[..., None] * 2.0
    assert (np.abs(got - out) <= (2.0 ** -8 + 2.0 ** -10 + slack) * spread + (2.0 ** -8 + slack) * np.abs(out)).all()
    assert (np.abs(r.lse[:r.rows].double().cpu().numpy() - lse) <= 2.0 ** -17 * size + 2.0 ** -22 * np.abs(lse) + 2.0 ** -14).all()


def test_requests_whose_blocks_do_not_suffice_are_left_out():
    r = Requests([(5, 60), (70, 100), (1, 64), (30, 0)], 7, 1, seed=2)
    r.prompts.n_blocks[1] = 2
    r.prompts.n_blocks[2] = 0
    before = r.k_cache.clone(), r.v_cache.clone()
    r.prepare()
    r.append()
    r.attend()
    torch.cuda.synchronize()
    for was, now in zip(before, (r.k_cache, r.v_cache)):
        for b in (1, 2):
            held = torch.from_numpy(r.table[b, :r.held[b]]).long()
            assert torch.equal(was[held].view(torch.int16), now[held].view(torch.int16))
    held = r.held
    r.k_cache.nan_to_num_(0.0), r.v_cache.nan_to_num_(0.0)       # (what the oracle reads of the requests that were left out)
    r.check(left_out=(1, 2))


def test_without_block_counts_and_without_lse():
    r = Requests([(33, 90), (1, 5)], 8, 2, seed=3, spare_columns=0)
    r.prompts.n_blocks, r.prompts.c.n_blocks = None, None
    r.prepare()
    r.append()
    r.attend(lse=None)
    torch.cuda.synchronize()
    assert (r.lse == 7.0).all()
    r.attend()
    r.check()


def test_table_entries_out_of_range_are_reported():
    r = Requests([(33, 90), (1, 5)], 8, 2, seed=3)
    r.prepare()
    r.append()
    torch.cuda.synchronize()
    r.prompts.block_table[0, 1] = r.num_blocks
    r.attend()
    torch.cuda.synchronize()
    assert int(r.status.item()) == sd.SD_ERR_BOUNDS
    r.status.zero_()
    r.prompts.block_table[0, 1] = -1
    r.prepare()
    torch.cuda.synchronize()
    assert int(r.status.item()) == sd.SD_ERR_BOUNDS


def test_repeats_bit_for_bit():
    r = Requests([(300, 50), (1, 2000), (1, 64), (90, 4000)], 28, 4, seed=9)
    r.prepare()
    r.append()
    r.attend()
    out, lse = r.out.clone(), r.lse.clone()
    for _ in range(3):
        r.prepare()
        r.attend()
        assert torch.equal(out.view(torch.int16), r.out.view(torch.int16)) and torch.equal(lse, r.lse)
    r.check()


def test_another_stream_and_a_captured_step():
    """Lengths that change between replays: the captured step follows what stands on the device."""
    r = Requests([(40, 100), (1, 300), (0, 0), (64, 0)], 7, 1, seed=4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    r.prepare(s)
    r.append(s)
    r.attend(s)
    s.synchronize()
    r.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.prepare()
        r.append()
        r.attend()
    r.out.fill_(7.0)
    r.lse.fill_(7.0)
    graph.replay()
    r.check()
    # fewer new tokens, in other requests
    r.new = np.array([10, 0, 0, 30], dtype=np.int32)
    r.len = np.array([100, 300, 0, 0], dtype=np.int32)
    rows = r.rows
    r.rows = 40
    r.prompts.n_new.copy_(torch.from_numpy(r.new))
    r.q[10:40], r.k[10:40], r.v[10:40] = r.q[41:71].clone(), r.k[41:71].clone(), r.v[41:71].clone()
    r.out.fill_(7.0)
    r.lse.fill_(7.0)
    graph.replay()
    r.check()
    assert rows > r.rows


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes, its last blocks in use."""
    lens = [(70, 300)]
    r = Requests(lens, 8, 8, seed=6, extra_rows=0)
    big = (1 << 32) // (8 * 64 * 128 * 2) + 9
    k, v = (torch.zeros((big, 8, 64, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    move = np.array([big - 1 - i for i in range(r.table.shape[1])], dtype=np.int32)
    for j in range(int(r.held[0])):
        k[move[j]], v[move[j]] = r.k_cache[r.table[0, j]], r.v_cache[r.table[0, j]]
    r.table = move[None]
    r.k_cache, r.v_cache, r.cache, r.num_blocks = k, v, sd.kv_layer(k, v), big
    r.prompts = sd.Prompts(r.N, 8, 8, 128, r.table, r.len, r.new, r.held, num_blocks=big)
    r.prepare()
    r.append()
    r.attend()
    torch.cuda.synchronize()
    small = torch.from_numpy(move[:int(r.held[0])]).long()
    r.k_cache, r.v_cache = k[small].clone(), v[small].clone()
    r.table = np.arange(int(r.held[0]), dtype=np.int32)[None]
    r.check()


def test_nothing_to_do():
    r = Requests([(0, 10), (0, 0)], 4, 2, seed=1, extra_rows=4)
    r.prepare()
    r.append()
    r.attend()
    r.check()
    empty = sd.Prompts(0, 4, 2, 128, r.table, r.len, r.new, r.held, num_blocks=r.num_blocks)
    sd.sd_prompt_prepare(empty, r.status)
    none = torch.empty((0, 4, 128), dtype=torch.bfloat16, device="cuda")
    sd.sd_append_kv(empty, r.cache, none[:, :2], none[:, :2], r.status)
    sd.sd_prompt_attention(empty, r.cache, none, r.scale, none, None, r.work, r.status)
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0 and empty.start.tolist() == [0, 0, 0]


@pytest.mark.parametrize("heads", [(4, 4), (7, 1)], ids=str)
def test_many_entries_of_one_tile(heads):
    """Thousands of entries that only one of the soft-max groups has a tile of, beside some of two and three."""
    g = np.random.default_rng(17)
    lens = [(1, int(c)) for c in g.integers(0, 64, 2000)] + [(1, int(c)) for c in g.integers(128, 300, 100)] + [(140, 0), (2, 127)]
    order = g.permutation(len(lens))
    r = Requests([lens[i] for i in order], *heads, seed=12)
    r.prepare()
    r.append()
    r.attend()
    r.check()


def test_a_plan_that_was_not_made_is_reported():
    r = Requests([(40, 100), (1, 300)], 7, 1, seed=4)
    r.prepare()
    r.append()
    torch.cuda.synchronize()
    for fill in (0, 255, 77):
        r.prompts.plan.fill_(fill)
        r.attend()
        torch.cuda.synchronize()
        assert int(r.status.item()) == sd.SD_ERR_INVALID_ARG and (r.out == 7.0).all() and (r.lse == 7.0).all()
        r.status.zero_()
    other = sd.Prompts(r.N - 2, 7, 1, 128, r.table, r.len, r.new, r.held, num_blocks=r.num_blocks)      # made for other sizes
    sd.sd_prompt_prepare(other, r.status)
    torch.cuda.synchronize()
    r.status.zero_()
    r.prompts.plan[:other.plan.numel()].copy_(other.plan)
    r.attend()
    torch.cuda.synchronize()
    assert int(r.status.item()) == sd.SD_ERR_INVALID_ARG and (r.out == 7.0).all()


@pytest.mark.parametrize("lens", [[(200, 3000)], [(1, 500)], [(30, 0), (1, 9)]], ids=str)
def test_waits_that_run_out_are_reported(lens, monkeypatch):
    r = Requests(lens, 7, 1, seed=4)
    r.prepare()
    r.append()
    torch.cuda.synchronize()
    monkeypatch.setenv("SDV_TEST_WITHHOLD", "1")
    monkeypatch.setenv("SDV_TEST_WAIT_CYCLES", "200000")
    r.attend()
    torch.cuda.synchronize()
    assert int(r.status.item()) == sd.SD_ERR_TIMEOUT
    monkeypatch.delenv("SDV_TEST_WITHHOLD")
    monkeypatch.delenv("SDV_TEST_WAIT_CYCLES")
    r.status.zero_()
    r.attend()                                               # and the next call finds everything as it should be
    r.check()


def test_objects_made_here_are_ready_on_any_stream():
    """Arrays that Prompts and BlockPool make on a busy stream, used at once on another, and dropped while that still runs."""
    side = torch.cuda.Stream()
    keep = Requests([(60, 10), (1, 90)], 7, 1, seed=6)
    torch.cuda.synchronize()
    for _ in range(5):
        torch.cuda._sleep(20000000)                          # the current stream is busy for some ten milliseconds
        p = sd.Prompts(keep.N, 7, 1, 128, keep.table.tolist(), keep.len.tolist(), keep.new.tolist(), keep.held.tolist(), num_blocks=keep.num_blocks)
        with torch.cuda.stream(side):
            torch.cuda._sleep(1000000)
        sd.sd_prompt_prepare(p, keep.status, side)
        sd.sd_append_kv(p, keep.cache, keep.k, keep.v, keep.status, side)
        sd.sd_prompt_attention(p, keep.cache, keep.q, keep.scale, keep.out, keep.lse, keep.work, keep.status, side)
        del p
        junk = [torch.full((1 << 16,), 2 ** 30, dtype=torch.int32, device="cuda") for _ in range(8)]
        torch.cuda.synchronize()
        del junk
        keep.check()
        keep.out.fill_(7.0)
        keep.lse.fill_(7.0)
    pool = sd.BlockPool(64)
    table, held, lens, new = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2, 8), (2,), (2,), (2,)))
    new += 100
    torch.cuda.synchronize()
    torch.cuda._sleep(20000000)
    pool = sd.BlockPool(64)
    sd.sd_assign_blocks(pool, table, held, lens, new, None, keep.status, side)
    torch.cuda.synchronize()
    assert table[:, :2].tolist() == [[0, 1], [2, 3]] and int(pool.n_free.item()) == 60


def test_arguments_that_do_not_fit_are_refused():
    r = Requests([(5, 3), (2, 0)], 4, 2, seed=1, extra_rows=0)
    r.prepare()
    bad = lambda **over: pytest.raises(AssertionError, r.attend, **over)
    bad(out=r.out[:, :3])
    bad(out=r.out.float())
    bad(lse=r.lse[:3])
    bad(out=torch.empty((r.N, 128, 4), dtype=torch.bfloat16, device="cuda").transpose(1, 2))
    bad(out=torch.empty((1, 4, 128), dtype=torch.bfloat16, device="cuda").expand(r.N, 4, 128))
    with pytest.raises(sd.SdError):
        r.attend(work=r.work[:-1])
    with pytest.raises(AssertionError):
        sd.sd_append_kv(r.prompts, r.cache, r.q, r.v, r.status)
    wide = torch.empty((r.N, 4, 132), dtype=torch.bfloat16, device="cuda")           # heads 132 apart, rows no multiple of 8
    with pytest.raises(AssertionError):
        r.attend(out=wide[:, :, :128])
    odd = torch.empty((r.N * 516 + 8,), dtype=torch.bfloat16, device="cuda")[:r.N * 516].view(r.N, 516)[:, :512].view(r.N, 4, 128)
    with pytest.raises(sd.SdError) as e:
        r.attend(out=odd)
    assert e.value.code == sd.SD_ERR_INVALID_ARG
    with pytest.raises(AssertionError):
        r.prompts.use(r.prompts.start, r.prompts.slot[:-1], r.prompts.position)
    with pytest.raises(AssertionError):
        r.prompts.use(r.prompts.start.long(), r.prompts.slot, r.prompts.position)
    with pytest.raises(AssertionError):
        sd.sd_assign_blocks(sd.BlockPool(8), r.prompts.block_table, r.prompts.n_blocks[:1], r.prompts.len, r.prompts.n_new, None, r.status)
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0


def test_two_calls_at_once():
    """Two layers on two streams, one plan, a workspace each: entries that are cut, joined by both."""
    a, c = (Requests([(1, 3000), (60, 900), (1, 17), (300, 0)], 14, 2, seed=8, gain=gain) for gain in (1.0, 3.0))
    a.prepare()
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        for r, s in zip((a, c), streams):
            sd.sd_append_kv(a.prompts, r.cache, r.k, r.v, r.status, s)
            sd.sd_prompt_attention(a.prompts, r.cache, r.q, r.scale, r.out, r.lse, r.work, r.status, s)
    a.check()
    c.check()


def test_two_captured_steps_share_a_workspace_one_after_the_other():
    a, c = (Requests([(1, 2000), (33, 500)], 7, 1, seed=s) for s in (1, 2))
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for r, g in ((a, graphs[0]), (c, graphs[1])):
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            r.prepare()
            r.append()
            r.attend(work=a.work)
    for g in graphs * 3:
        g.replay()
    a.check()
    c.check()


def test_a_prefix_that_requests_share():
    """Blocks that several tables name are read by all of them."""
    r = Requests([(5, 256), (70, 300), (1, 700)], 8, 2, seed=6)
    r.table[1, :4] = r.table[0, :4]
    r.table[2, :4] = r.table[0, :4]
    r.prompts.block_table.copy_(torch.from_numpy(r.table))
    r.prepare()
    r.append()
    r.attend()
    r.check()


def test_tables_that_would_be_taken_wrongly_are_refused():
    make = lambda table, lens=(1, 2): sd.Prompts(3, 4, 2, 128, table, list(lens), [1, 2], num_blocks=8)
    wide = torch.zeros((2, 6), dtype=torch.int32, device="cuda")
    for bad in (wide[:, :4], wide.reshape(4, 3), wide.reshape(12)):          # a copy would not follow; four sequences; no rows
        with pytest.raises(AssertionError):
            make(bad)
    assert make(wide).block_table is wide
    assert make(wide[:, :4].long()).max_blocks == 4                          # (another type: copied in any case)


@pytest.mark.parametrize("heads", [(64, 64), (128, 64), (4, 2)], ids=str)
def test_spikes_and_plateaus(heads):
    """Single keys that tower over all others, and stretches just below them: weights that were relative to the reference before the spike, in the tile
    behind it and in the other half of its own, are brought to the one after it.  (So many heads that a CTA has whole entries; few, and they are cut.)"""
    g = np.random.default_rng(21)
    r = Requests([(20, 900), (3, 700), (1, 1200), (129, 500), (20, 640), (64, 300), (20, 128), (1, 2000), (33, 1000), (20, 1100)], *heads, seed=21)
    r.prepare()
    r.append()
    r.q[:r.rows] = 1.0
    for b, (n, c) in enumerate(r.lens):
        level = g.normal(0.0, 1.0, n + c)                                       # in powers of two
        for t0 in range(0, n + c, 64):
            stretch = slice(t0, min(t0 + 64, n + c))
            level[stretch] += g.choice([0.0, 0.0, 20.0, 31.0])
            if g.random() < 0.4:
                level[g.integers(t0, min(t0 + 64, n + c))] = g.choice([35.0, 45.0, 80.0, 120.0]) + 3.0 * b
        values = torch.from_numpy((level * np.log(2.0) * np.sqrt(128.0) / 128.0).astype(np.float32)).to(torch.bfloat16).cuda()
        t = torch.arange(n + c, device="cuda")
        block = torch.from_numpy(r.table[b]).cuda().long()[t // 64]
        r.k_cache[block, :, t % 64] = values[:, None, None].expand(-1, heads[1], 128)
    r.attend()
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0
    out, lse, spread, size = r.expect()
    got = r.out[:r.rows].double().cpu().numpy()
    slack = 2.0 ** -17 * size[..., None] * 2.0
    assert (np.abs(got - out) <= (2.0 ** -8 + 2.0 ** -10 + slack) * spread + (2.0 ** -8 + slack) * np.abs(out)).all()
    assert (np.abs(r.lse[:r.rows].double().cpu().numpy() - lse) <= 2.0 ** -17 * size + 2.0 ** -22 * np.abs(lse) + 2.0 ** -14).all()
