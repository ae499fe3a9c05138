"""GPU: block tables from lengths, slots of packed tokens, K/V into their slots; whole numbers and bytes against the oracle."""
import numpy as np
import pytest
import torch

from oracle import prompt as ref
from paper_2509_18824_b200 import binding as sd
from prompt_util import Requests, blocks

pytestmark = pytest.mark.gpu


def to(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


class Pages:
    """B requests that hold blocks for `held_tokens`, in tables of W entries; a pool with `spare` more."""

    def __init__(self, held_tokens, W, spare, seed=0):
        g = np.random.default_rng(seed)
        self.held = np.array([blocks(int(t)) for t in held_tokens], dtype=np.int32)
        self.num_blocks = int(self.held.sum()) + spare
        order = g.permutation(self.num_blocks).astype(np.int32)
        self.table = np.full((len(self.held), W), -7, dtype=np.int32)
        at = 0
        for b, h in enumerate(self.held):
            self.table[b, :h] = order[at:at + h]
            at += h
        self.stack = np.concatenate([order[at:], np.full(at, -9, dtype=np.int32)])
        self.n_free = spare
        self.d_table, self.d_held = to(self.table), to(self.held)
        self.pool = sd.BlockPool(self.num_blocks, to(self.stack), to([self.n_free]))
        self.granted = torch.full((len(self.held),), -3, dtype=torch.int32, device="cuda")
        self.status = sd.new_status()

    def call(self, lens, new, stream=None):
        sd.sd_assign_blocks(self.pool, self.d_table, self.d_held, to(lens), to(new), self.granted, self.status, stream)

    def check(self, lens, new):
        self.table, self.held, self.stack, self.n_free, granted = ref.assign(self.table, self.held, lens, new, self.stack, self.n_free)
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        for got, want in ((self.d_table, self.table), (self.d_held, self.held), (self.granted, granted), (self.pool.n_free, [self.n_free])):
            np.testing.assert_array_equal(got.cpu().numpy(), want)
        np.testing.assert_array_equal(self.pool.free_blocks.cpu().numpy()[:self.n_free], self.stack[:self.n_free])
        owned = np.concatenate([self.table[b, :h] for b, h in enumerate(self.held)] + [self.stack[:self.n_free]])
        assert np.array_equal(np.sort(owned), np.arange(self.num_blocks))          # every block has one owner


@pytest.mark.parametrize("B", [1, 2, 31, 64, 65, 300, 1024, 1025, 5000])
@pytest.mark.parametrize("spare", [0, 7, 100000])
def test_tables_follow_lengths(B, spare):
    g = np.random.default_rng(B + spare)
    longest = 6400 if B < 2000 else 640
    lens = g.integers(0, longest, B)
    lens[g.random(B) < 0.2] = 0
    p = Pages(lens, blocks(longest) + 40, min(spare, 40 * B + 5), seed=B)
    for step in range(4):
        new = g.integers(0, 200, B) * (g.random(B) < 0.7)
        new[g.random(B) < 0.05] = 2000
        done = g.random(B) < 0.1
        lens, new = np.where(done, 0, lens), np.where(done, 0, new)
        p.call(lens, new)
        p.check(lens, new)
        took = p.granted.cpu().numpy() == 1
        lens = np.where(took, np.minimum(lens + g.integers(0, 70, B), lens + new), np.minimum(lens, 64 * p.held))


def test_giving_back_what_was_taken_restores_the_pool():
    g = np.random.default_rng(3)
    lens = g.integers(0, 3000, 200)
    p = Pages(lens, 80, 500, seed=1)
    held, stack = p.held.copy(), p.stack.copy()
    for _ in range(3):
        p.call(lens, np.full(200, 100))
        p.check(lens, np.full(200, 100))
        p.call(lens, np.zeros(200))
        p.check(lens, np.zeros(200))
        np.testing.assert_array_equal(p.held, held)
        np.testing.assert_array_equal(p.pool.free_blocks.cpu().numpy(), stack)


def test_requests_in_front_of_a_short_one_are_served_and_none_behind_it():
    p = Pages([64, 64, 64, 64], 10, 3, seed=2)
    lens, new = np.array([64, 64, 64, 64]), np.array([100, 300, 10, 0])      # need 2, 5, 1, 0 of 3
    p.call(lens, new)
    p.check(lens, new)
    assert p.granted.tolist() == [1, 0, 0, 1] and int(p.pool.n_free.item()) == 1


@pytest.mark.parametrize("B", [5, 90])
def test_bad_lengths_and_counts_are_reported_and_change_nothing_of_theirs(B):
    for what, code in (("len", sd.SD_ERR_INVALID_ARG), ("new", sd.SD_ERR_INVALID_ARG), ("too_long", sd.SD_ERR_BOUNDS), ("held", sd.SD_ERR_BOUNDS),
                       ("held_high", sd.SD_ERR_BOUNDS), ("huge", sd.SD_ERR_BOUNDS)):
        p = Pages([100] * B, 6, 20, seed=4)
        lens, new = np.full(B, 100), np.zeros(B, dtype=np.int64)
        new[0] = 100
        if what == "len":
            lens[2] = -1
        elif what == "new":
            new[2] = -5
        elif what == "too_long":
            new[2] = 300
        elif what == "huge":
            lens[2] = new[2] = 2 ** 31 - 1
        else:
            p.d_held[2] = -1 if what == "held" else 7
        p.call(lens, new)
        torch.cuda.synchronize()
        assert int(p.status.item()) == code, what
        held = p.d_held.cpu().numpy()
        assert held[0] == 4 and held[1] == 2 and held[2] == {"held": -1, "held_high": 7}.get(what, 2)
        np.testing.assert_array_equal(p.d_table.cpu().numpy()[2], p.table[2])
        assert int(p.pool.n_free.item()) == 18


def test_a_pool_that_overflows_or_counts_wrongly_is_reported():
    p = Pages([200, 200], 6, 4, seed=4)
    p.pool.n_free.fill_(p.num_blocks)                        # blocks that are held count as free as well: they come back a second time
    p.call(np.zeros(2), np.zeros(2))
    torch.cuda.synchronize()
    assert int(p.status.item()) == sd.SD_ERR_BOUNDS and int(p.pool.n_free.item()) == p.num_blocks
    for n in (-1, p.num_blocks + 1):
        p = Pages([64, 64], 6, 4, seed=4)
        p.pool.n_free.fill_(n)
        p.call(np.array([64, 64]), np.array([64, 0]))
        torch.cuda.synchronize()
        assert int(p.status.item()) == sd.SD_ERR_BOUNDS and p.granted.tolist() == [0, 1] and p.d_held.tolist() == [1, 1]


@pytest.mark.parametrize("extra", [0, 1, 5000])
@pytest.mark.parametrize("kind", ["mixed", "singles", "long", "many"])
def test_slots_and_positions(kind, extra):
    g = np.random.default_rng(7)
    lens = {"mixed": [(int(g.integers(0, 300)), int(g.integers(0, 500))) for _ in range(50)], "singles": [(1, int(c)) for c in g.integers(0, 900, 70)],
            "long": [(9000, 0), (3, 5000)], "many": [(int(g.integers(0, 4)), int(g.integers(0, 70))) for _ in range(3000)]}[kind]
    r = Requests(lens, 1, 1, seed=11, extra_rows=extra)
    short = [b for b in range(len(lens)) if b % 7 == 3]
    r.held[short] = np.maximum(r.held[short] - 1, 0)
    r.prompts.n_blocks.copy_(to(r.held))
    r.prepare()
    start, slot, position = ref.slots(r.table, r.held, r.len, r.new, r.N)
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0
    np.testing.assert_array_equal(r.prompts.start.cpu().numpy(), start)
    np.testing.assert_array_equal(r.prompts.slot.cpu().numpy(), slot)
    np.testing.assert_array_equal(r.prompts.position.cpu().numpy(), position)


def test_more_new_tokens_than_rows_are_reported():
    r = Requests([(5, 0), (9, 0)], 1, 1, extra_rows=0)
    r.prompts.n_new[0] = 6
    r.prepare()
    torch.cuda.synchronize()
    assert int(r.status.item()) == sd.SD_ERR_BOUNDS
    assert r.prompts.start.tolist() == [0, 6, 14] and (r.prompts.slot[6:] == -1).all()
    for bad in ("n_new", "len"):
        r = Requests([(5, 0), (9, 0)], 1, 1, extra_rows=0)
        getattr(r.prompts, bad)[0] = -2
        r.prepare()
        torch.cuda.synchronize()
        assert int(r.status.item()) == sd.SD_ERR_INVALID_ARG and (r.prompts.slot[:0 if bad == "n_new" else 5] == -1).all()


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("heads", [(1, 1), (28, 4), (3, 3), (8, 8)], ids=str)
def test_rows_reach_their_slots_and_nothing_else_changes(heads, strided):
    r = Requests([(1, 63), (200, 5), (0, 9), (64, 64), (1, 0)], *heads, seed=3, strided=strided)
    want = [c.view(torch.int16).cpu().numpy().copy() for c in (r.k_cache, r.v_cache)]
    _, slot, _ = ref.slots(r.table, r.held, r.len, r.new, r.N)
    for cache, rows in zip(want, (r.k, r.v)):
        x = rows.contiguous().view(torch.int16).cpu().numpy()
        for i, s in enumerate(slot):
            if s >= 0:
                cache[s // 64, :, s % 64] = x[i]
    r.prepare()
    r.append()
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0
    for cache, w in zip((r.k_cache, r.v_cache), want):
        np.testing.assert_array_equal(cache.view(torch.int16).cpu().numpy(), w)


@pytest.mark.parametrize("B", [3, 400])
def test_requests_out_of_range_are_not_granted(B):
    p = Pages([100] * B, 6, 20, seed=4)
    lens, new = np.full(B, 100), np.zeros(B, dtype=np.int64)
    lens[1], new[0] = 400, 100                               # seven blocks of six; four
    p.call(lens, new)
    torch.cuda.synchronize()
    assert int(p.status.item()) == sd.SD_ERR_BOUNDS
    assert p.granted.tolist() == [1, 0] + [1] * (B - 2) and p.d_held.tolist() == [4] + [2] * (B - 1)


@pytest.mark.parametrize("bad", [-1, 24, 2 ** 30])
def test_blocks_out_of_range_that_change_hands_are_reported(bad):
    p = Pages([100, 100], 6, 20, seed=4)
    p.d_table[1, 1] = bad                                    # given back
    p.call(np.array([100, 0]), np.zeros(2))
    torch.cuda.synchronize()
    assert int(p.status.item()) == sd.SD_ERR_BOUNDS and int(p.pool.n_free.item()) == 22
    p.status.zero_()
    p.call(np.array([100, 100]), np.zeros(2))                # and taken
    torch.cuda.synchronize()
    assert int(p.status.item()) == sd.SD_ERR_BOUNDS and p.d_table[1, 1].item() == bad


def test_the_most_requests():
    B = 8192
    g = np.random.default_rng(9)
    lens, new = g.integers(0, 300, B), g.integers(0, 4, B)
    p = Pages(lens, 8, 12000, seed=9)
    p.call(lens, new)
    p.check(lens, new)
    N = int(new.sum()) + 5
    q = sd.Prompts(N, 2, 1, 128, p.d_table, lens, new, p.d_held, num_blocks=p.num_blocks)
    sd.sd_prompt_prepare(q, p.status)
    torch.cuda.synchronize()
    assert int(p.status.item()) == 0
    for got, want in zip((q.start, q.slot, q.position), ref.slots(p.table, p.held, lens, new, N)):
        np.testing.assert_array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("B, Hkv, tokens", [(40, 8, 100000), (3, 64, 2 ** 24), (1500, 4, 2 ** 19), (1, 2, 10 ** 6)])
def test_parts_are_equal_however_long(B, Hkv, tokens):
    """Single tokens behind long contexts: where the CTAs' parts begin, as the plan's words say it (entries of key tiles and two more)."""
    g = np.random.default_rng(B)
    lens = tokens - g.integers(0, tokens // 2, B) - 1
    if B > 1000:
        lens[1:] = g.integers(0, 200, B - 1)                 # (that many of one length would be dealt out)
    W = blocks(tokens)
    q = sd.Prompts(B, Hkv, Hkv, 128, torch.zeros((B, W), dtype=torch.int32, device="cuda"), lens, np.ones(B, dtype=np.int32), num_blocks=1)
    st = sd.new_status()
    sd.sd_prompt_prepare(q, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    words = q.plan.cpu().numpy()[:16 + 48 * (sms + 1)].view(np.int32)
    assert words[1] == 0                                     # in parts
    starts = words[4:].reshape(sms + 1, 12)[:, :3].astype(np.int64)
    one = -(-(lens // 64 + 1) // 2) + 2
    before = np.concatenate([[0], np.cumsum(one)]) * Hkv
    line = int(before[-1])
    part = -(-line // sms)
    e, h, tile = starts.T
    assert tuple(starts[-1]) == (B, 0, 0)
    at = before[e] + h * np.append(one, 0)[e] + np.where(tile > 0, tile + 2, 0)
    want = np.minimum(np.arange(sms + 1) * part, line)
    assert np.abs(at - want).max() <= 6 and (np.diff(at) > 0).all()


@pytest.mark.parametrize("B, new, heads", [(200, 2000, (8, 1)), (300, 40, (28, 4)), (2000, 50, (28, 4)), (8, 4096, (28, 4)), (700, 1, (64, 64))], ids=str)
def test_entries_that_are_dealt_out_stand_in_order(B, new, heads):
    """Every row tile once, the longest first, and each CTA's first piece in its start."""
    g = np.random.default_rng(B)
    lens, n = g.integers(0, 3000, B), g.integers(0, new + 1, B)
    n[0] = new
    W, N = blocks(3000 + new), int(n.sum())
    q = sd.Prompts(N, *heads, 128, torch.zeros((B, W), dtype=torch.int32, device="cuda"), lens, n, num_blocks=1)
    st = sd.new_status()
    sd.sd_prompt_prepare(q, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    tokens = 128 // (heads[0] // heads[1])
    row0 = np.concatenate([[0], np.cumsum(n)])
    want = [(row0[b] + i, lens[b] + i, min(tokens, n[b] - i), b, blocks(int(lens[b] + min(i + tokens, n[b]))), lens[b] + n[b])
            for b in range(B) for i in range(0, int(n[b]), tokens)]
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    raw = q.plan.cpu().numpy()
    words = lambda at, count: raw[at:at + 4 * count].view(np.int32)
    entries = int(words(0, 4)[1])
    assert entries == len(want)
    starts, at = words(16, 12 * (sms + 1)).reshape(-1, 12), 16 + 48 * (sms + 1) + 32 * sms
    cap = N // tokens + min(B, N) + 1
    got = words(at, 8 * entries).reshape(-1, 8)[:, :6]
    np.testing.assert_array_equal(got, np.array(want))
    order = words(at + 32 * cap, entries)
    assert np.array_equal(np.sort(order), np.arange(entries))
    tiles = (got[:, 4] + 1) // 2
    assert (np.diff(tiles[order]) <= 0).all()
    for c in range(min(sms, entries * heads[1])):
        assert tuple(starts[c, :2]) == (c, c % heads[1])
        np.testing.assert_array_equal(starts[c, 4:10], got[order[c // heads[1]]])
