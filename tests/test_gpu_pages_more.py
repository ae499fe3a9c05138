"""GPU: slots, positions and attention beside requests whose numbers are out of range; geometries at the limits of what is accepted."""
import numpy as np
import pytest
import torch

from oracle import prompt as ref
from paper_2509_18824_b200 import binding as sd
from prompt_util import Requests, blocks

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["n_new", "len"])
def test_requests_beside_one_whose_numbers_are_negative(what):
    r = Requests([(5, 70), (9, 0), (30, 100)], 4, 2, seed=3, extra_rows=4)
    bad = r.prompts.n_new if what == "n_new" else r.prompts.len
    bad[0] = -2
    r.prepare()
    torch.cuda.synchronize()
    assert int(r.status.item()) == sd.SD_ERR_INVALID_ARG
    r.status.zero_()
    # without the bad request: its rows are nobody's (no tokens), or left out (no length)
    new = np.array([0 if what == "n_new" else 5, 9, 30])
    start = np.concatenate([[0], np.cumsum(new)])
    slot, position = np.full(r.N, -1), np.zeros(r.N, dtype=np.int64)
    for b in (1, 2):
        t = int(r.len[b]) + np.arange(new[b])
        slot[start[b]:start[b + 1]] = r.table[b, t // 64] * 64 + t % 64
        position[start[b]:start[b + 1]] = t
    np.testing.assert_array_equal(r.prompts.start.cpu().numpy(), start)
    np.testing.assert_array_equal(r.prompts.slot.cpu().numpy(), slot)
    rest = np.ones(r.N, dtype=bool)
    rest[:start[1]] = False                                  # (rows of a request without a length have no place that means anything)
    np.testing.assert_array_equal(r.prompts.position.cpu().numpy()[rest], position[rest])
    # and the attention of the others
    finite = torch.nan_to_num(r.q, 0.0), torch.nan_to_num(r.k, 0.0), torch.nan_to_num(r.v, 0.0)
    r.q, r.k, r.v = (x.contiguous() for x in finite)
    r.append()
    r.attend()
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0
    d = lambda t: t.double().cpu().numpy()
    for b in (1, 2):
        rows = slice(int(start[b]), int(start[b + 1]))
        want, want_lse, spread, _ = ref.attention(d(r.q[rows]), d(r.k_cache), d(r.v_cache), r.table[b:b + 1], r.len[b:b + 1], new[b:b + 1], r.scale)
        assert (np.abs(d(r.out[rows]) - want) <= (2.0 ** -8 + 2.0 ** -10) * spread + 2.0 ** -8 * np.abs(want)).all()
        assert (np.abs(d(r.lse[rows]) - want_lse) <= 2.0 ** -12).all()
    untouched = torch.ones(r.N, dtype=torch.bool, device="cuda")
    untouched[int(start[1]):int(start[3])] = False
    assert (r.out[untouched] == 7.0).all() and (r.lse[untouched] == 7.0).all()


@pytest.mark.parametrize("heads", [(1024, 128), (1024, 1024), (1000, 200), (1, 1)], ids=str)
def test_the_most_and_fewest_heads(heads):
    r = Requests([(3, 130), (1, 64), (17, 0)], *heads, seed=2)
    r.prepare()
    r.append()
    r.attend()
    r.check()


def test_many_rows_of_nobody():
    r = Requests([(0, 5), (70, 10), (1, 300), (0, 0)], 14, 2, seed=2, extra_rows=20000)
    r.prepare()
    r.append()
    r.attend()
    r.check()


def test_two_plans_at_once():
    """Two batches on two streams, everything their own but the caches' kernels."""
    a, b = Requests([(200, 500), (1, 3000)], 8, 2, seed=5), Requests([(1, c) for c in range(0, 3000, 111)], 8, 2, seed=6)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        for r, s in zip((a, b), streams):
            r.prepare(s)
            r.append(s)
            r.attend(s)
    a.check()
    b.check()


@pytest.mark.parametrize("tokens", [1 << 20, (1 << 24) + 77])
def test_very_long_contexts_over_blocks_that_repeat(tokens):
    """A table that names one block over and over: the values' weighted mean is that of one block (and the last one's share), whatever the length."""
    g = np.random.default_rng(4)
    W = blocks(tokens + 1)
    k, v = (torch.randn((2, 1, 64, 128), device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.zeros((1, W), dtype=torch.int32, device="cuda")
    table[0, W - 1] = 1
    q = torch.randn((1, 4, 128), device="cuda").to(torch.bfloat16)
    p = sd.Prompts(1, 4, 1, 128, table, [tokens], [1], num_blocks=2)
    st, out, lse = sd.new_status(), torch.zeros((1, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 4), device="cuda")
    work = torch.empty(sd.sd_prompt_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    sd.sd_prompt_prepare(p, st)
    sd.sd_append_kv(p, sd.kv_layer(k, v), torch.randn((1, 1, 128), device="cuda").to(torch.bfloat16), torch.randn((1, 1, 128), device="cuda").to(torch.bfloat16), st)
    sd.sd_prompt_attention(p, sd.kv_layer(k, v), q, 0.1, out, lse, work, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    d = lambda t: t.double().cpu().numpy()
    last = tokens - 64 * (W - 1) + 1
    keys, values = np.concatenate([d(k)[0, 0], d(k)[1, 0, :last]]), np.concatenate([d(v)[0, 0], d(v)[1, 0, :last]])
    times = np.concatenate([np.full(64, W - 1.0), np.ones(last)])
    z = 0.1 * d(q)[0] @ keys.T
    e = np.exp(z - z.max(axis=1, keepdims=True)) * times
    want, spread = e @ values / e.sum(axis=1)[:, None], e @ np.abs(values) / e.sum(axis=1)[:, None]
    # sums of so many terms in 32 bits: each of the additions of a CTA's share rounds by at most 2^-24 of what is there (the sum's) or
    # cuts 2^-23 (the products'); every 16 keys one
    adds = 2.0 ** -23 * (tokens / 16 / torch.cuda.get_device_properties(0).multi_processor_count + 64)
    assert (np.abs(d(out)[0] - want) <= (2.0 ** -8 + 2.0 ** -10 + adds) * spread + 2.0 ** -8 * np.abs(want)).all()
    assert (np.abs(d(lse)[0] - np.log(e.sum(axis=1)) - z.max(axis=1)) <= 2.0 ** -12 + adds).all()
