"""GPU: attention of packed tokens gives the same bits in every run, also where rows' references are raised: in an entry's first tile, while the
other soft-max group takes the second one up, and later."""
import numpy as np
import pytest
import torch

from prompt_util import Requests

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["first_tile", "spikes", "rising"])
@pytest.mark.parametrize("heads", [(64, 64), (128, 64), (4, 2), (7, 1)], ids=str)       # (many: entries are whole; few: they are cut)
def test_raised_references_repeat_bit_for_bit(heads, kind):
    g = np.random.default_rng(31)
    lens = [(20, 900), (3, 700), (1, 1200), (129, 500), (64, 300), (20, 128), (1, 2000), (33, 1000), (130, 0), (5, 130)]
    r = Requests(lens, *heads, seed=31)
    r.prepare()
    r.append()
    # scores: one power of two for all rows, by key, and what differs from row to row
    r.q[:r.rows] = 1.0 + 0.25 * torch.rand((r.rows, heads[0], 1), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    for b, (n, c) in enumerate(lens):
        level = g.normal(0.0, 1.0, n + c)
        if kind == "first_tile":
            for t0 in range(0, n + c, 128):                                     # (also of every chunk)
                level[min(t0 + 40 + 3 * b, n + c - 1)] = 50.0
                level[t0:t0 + 32] -= 20.0
        elif kind == "spikes":
            for t0 in range(0, n + c, 64):
                if g.random() < 0.5:
                    level[g.integers(t0, min(t0 + 64, n + c))] = g.choice([35.0, 45.0, 80.0, 120.0])
        else:
            level += 40.0 * (np.arange(n + c) // 64)
        values = torch.from_numpy((level * np.log(2.0) * np.sqrt(128.0) / 128.0).astype(np.float32)).to(torch.bfloat16).cuda()
        t = torch.arange(n + c, device="cuda")
        block = torch.from_numpy(r.table[b]).cuda().long()[t // 64]
        r.k_cache[block, :, t % 64] = values[:, None, None].expand(-1, heads[1], 128)
    r.attend()
    torch.cuda.synchronize()
    assert int(r.status.item()) == 0
    out, lse = r.out.clone(), r.lse.clone()
    want, want_lse, spread, size = r.expect()
    got = r.out[:r.rows].double().cpu().numpy()
    slack = 2.0 ** -17 * size[..., None] * 2.0              # (128 products of this size: a score is off by up to 2^-17 of it)
    assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -10 + slack) * spread + (2.0 ** -8 + slack) * np.abs(want)).all()
    assert (np.abs(r.lse[:r.rows].double().cpu().numpy() - want_lse) <= 2.0 ** -17 * size + 2.0 ** -22 * np.abs(want_lse) + 2.0 ** -14).all()
    for _ in range(100):
        r.attend()
        assert torch.equal(out.view(torch.int16), r.out.view(torch.int16)) and torch.equal(lse, r.lse)
    assert int(r.status.item()) == 0
