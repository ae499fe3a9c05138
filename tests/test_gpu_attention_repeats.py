"""GPU: tree attention gives the same bits in every run, also where rows' references are raised: in the first tile, while the other soft-max
group takes the second one up, and later."""
import numpy as np
import pytest
import torch

import oracle
from paper_2509_18824_b200 import workloads as wl
from paper_2509_18824_b200.step import VerifyStep
from gpu_util import check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["first_tile", "spikes", "rising"])
@pytest.mark.parametrize("B, prefix, T", [(1, 2000, 60), (3, 700, 60), (24, 200, 11), (16, 900, 28)])
def test_raised_references_repeat_bit_for_bit(B, prefix, T, kind):
    g = np.random.default_rng(B)
    w = wl.make("c5", B=B, L=1, V=64, Hd=64, prefix=prefix, T=T)
    one = wl.f32_to_bf16_bits(1.0 + 0.25 * g.random(w.q[0].shape[:3] + (1,)).astype(np.float32))
    w.q[0][:] = one
    for b in range(B):
        level = g.normal(0.0, 1.0, prefix)
        if kind == "first_tile":
            for t0 in range(0, prefix, 64):                  # (of every chunk, wherever it begins)
                level[t0:t0 + 16] -= 20.0
                # far above them; below the sum that raises by itself; and as before
                level[min(t0 + 20 + b, prefix - 1)] = [50.0, 12.0, 14.5][(t0 // 64) % 3]
        elif kind == "spikes":
            for t0 in range(0, prefix, 64):
                if g.random() < 0.5:
                    level[g.integers(t0, min(t0 + 64, prefix))] = g.choice([35.0, 45.0, 80.0, 120.0])
        else:
            level += 40.0 * (np.arange(prefix) // 64)
        bits = wl.f32_to_bf16_bits((level * np.log(2.0) / (float(w.scale) * 128.0)).astype(np.float32))
        t = np.arange(prefix)
        w.k_cache[0][w.block_table[b, t // 64], :, t % 64] = bits[:, None, None]
    vs = VerifyStep(w)
    vs.attention(0)
    torch.cuda.synchronize()
    vs.check_status()
    out, lse = vs.out[0].clone(), vs.lse[0].clone()
    want, _ = oracle.attention(oracle.Geometry.of(w), w.k_cache[0], w.v_cache[0], w.q[0], w.k_tree[0], w.v_tree[0], w.scale)
    check_attention(out.float().cpu().numpy(), want)
    for i in range(100):
        vs.attention(0) if i % 2 else vs.attention_layers()
        assert torch.equal(out.view(torch.int16), vs.out[0].view(torch.int16)) and torch.equal(lse, vs.lse[0])
    vs.check_status()
