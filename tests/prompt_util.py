"""Packed new tokens for the tests of the calls on them: requests on the device, comparison with the oracle."""
import numpy as np
import torch

from oracle import prompt as ref
from paper_2509_18824_b200 import binding as sd


def blocks(tokens):
    return -(-tokens // 64)


class Requests:
    """Requests [(new, cached)] over a shuffled pool; everything that no request's tokens fill is NaN: blocks of nobody, slots behind the
    last token, packed rows of nobody, and what lies between strided rows."""

    def __init__(self, lens, Hq, Hkv, seed=0, extra_rows=3, spare_columns=2, strided=True, gain=2.0):
        g = np.random.default_rng(seed)
        self.lens, self.Hq, self.Hkv = lens, Hq, Hkv
        self.new, self.len = (np.array([p[i] for p in lens], dtype=np.int32) for i in (0, 1))
        self.rows = int(self.new.sum())
        self.N = self.rows + extra_rows
        held = np.array([blocks(n + c) for n, c in lens], dtype=np.int32)
        W = max(1, int(held.max())) + spare_columns
        self.num_blocks = int(held.sum()) + 3
        order = g.permutation(self.num_blocks).astype(np.int32)
        self.table = np.full((len(lens), W), 2 ** 30, dtype=np.int32)
        at = 0
        for b, h in enumerate(held):
            self.table[b, :h] = order[at:at + h]
            at += h
        self.held = held
        bf = lambda a: torch.from_numpy(a.astype(np.float32)).to(torch.bfloat16).cuda()
        ld = Hq + 2 * Hkv + (1 if strided else 0)
        whole = torch.full((self.N, ld, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
        whole[:self.rows, :Hq + 2 * Hkv] = bf(g.standard_normal((self.rows, Hq + 2 * Hkv, 128)))
        whole[:self.rows, :Hq] *= gain
        if strided:
            self.q, self.k, self.v = whole[:, :Hq], whole[:, Hq:Hq + Hkv], whole[:, Hq + Hkv:Hq + 2 * Hkv]
        else:
            self.q, self.k, self.v = (x.contiguous() for x in (whole[:, :Hq], whole[:, Hq:Hq + Hkv], whole[:, Hq + Hkv:]))
        shape = (self.num_blocks, Hkv, 64, 128)
        self.k_cache, self.v_cache = (torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        for b, (n, c) in enumerate(lens):
            for j in range(blocks(c)):
                m = min(c - 64 * j, 64)
                for cache in (self.k_cache, self.v_cache):
                    cache[self.table[b, j], :, :m] = bf(g.standard_normal((Hkv, m, 128)))
        self.scale = 1.0 / np.sqrt(128.0)
        self.status = sd.new_status()
        self.prompts = sd.Prompts(self.N, Hq, Hkv, 128, self.table, self.len, self.new, self.held, num_blocks=self.num_blocks)
        self.cache = sd.kv_layer(self.k_cache, self.v_cache)
        self.work = torch.empty(sd.sd_prompt_workspace_bytes(self.prompts), dtype=torch.uint8, device="cuda").fill_(255)
        out = torch.full((self.N, Hq + (1 if strided else 0), 128), 7.0, dtype=torch.bfloat16, device="cuda")
        self.out = out[:, :Hq]
        self.lse = torch.full((self.N, Hq), 7.0, device="cuda")

    def prepare(self, stream=None):
        sd.sd_prompt_prepare(self.prompts, self.status, stream)

    def append(self, stream=None):
        sd.sd_append_kv(self.prompts, self.cache, self.k, self.v, self.status, stream)

    def attend(self, stream=None, **over):
        a = dict(out=self.out, lse=self.lse, work=self.work)
        a.update(over)
        sd.sd_prompt_attention(self.prompts, self.cache, self.q, self.scale, a["out"], a["lse"], a["work"], self.status, stream)

    def expect(self):
        d = lambda t: t.double().cpu().numpy()
        return ref.attention(d(self.q)[:self.rows], d(self.k_cache), d(self.v_cache), self.table, self.len, self.new, self.scale)

    def check(self, want=None, left_out=()):
        """out and lse against the oracle.  A weight is rounded to bf16 (half a step, 2^-8), the output too; the rest is fp32: 128 products
        in a score (2^-24 of their size each), the row's sum, the exponential (2^-22): together below 2^-10 of the weights at these sizes."""
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        out, lse, spread, size = self.expect() if want is None else want
        got, got_lse = self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()
        start = np.concatenate([[0], np.cumsum(self.new)])
        keep = np.ones(self.rows, dtype=bool)
        for b in left_out:
            keep[start[b]:start[b + 1]] = False
        keys = int((self.new + self.len).max())
        assert 2.0 ** -24 * (128 * size.max(initial=0.0) + keys) < 2.0 ** -10
        bound = (2.0 ** -8 + 2.0 ** -10) * spread + 2.0 ** -8 * np.abs(out) + 1e-30
        err = np.abs(got[:self.rows] - out)[keep]
        assert np.isfinite(got[:self.rows][keep]).all()
        worst = float((err / bound[keep]).max()) if err.size else 0.0
        assert worst <= 1.0, worst
        bound_lse = 2.0 ** -24 * (128 * size + keys + 64) + 2.0 ** -22 * np.abs(lse)
        err = np.abs(got_lse[:self.rows] - lse)[keep]
        assert not err.size or float((err / bound_lse[keep]).max()) <= 1.0, float((err / bound_lse[keep]).max())
        # rows of nobody, of requests that were left out, and between the rows: as they were
        assert (got[self.rows:] == 7.0).all() and (got_lse[self.rows:] == 7.0).all()
        assert (got[:self.rows][~keep] == 7.0).all() and (got_lse[:self.rows][~keep] == 7.0).all()
        base = self.out._base
        if base is not None and base.shape[1] > self.Hq:
            assert (base[:, self.Hq:] == 7.0).all()
        return worst
