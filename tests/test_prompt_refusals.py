"""Argument checks of the calls on packed new tokens: refused on the host, before any launch (no GPU here); the oracle's own pins."""
import ctypes

import numpy as np
import pytest

from oracle import prompt as ref
from paper_2509_18824_b200 import binding as b

f = ctypes.c_float
ok = 4096                                                   # any 16-byte aligned, non-null stand-in address


def prompts(B=2, N=10, Hq=8, Hkv=2, D=128, block=64, W=4, blocks=8, table=ok, n_blocks=ok, lens=ok, new=ok, start=ok, slot=ok, pos=ok, plan=ok):
    return b.sd_prompts(B, N, Hq, Hkv, D, block, W, blocks, table, n_blocks, lens, new, start, slot, pos, plan)


def prepare(st=ok, **over):
    return b.lib.sd_prompt_prepare(ctypes.byref(prompts(**over)), st, None)


def append(k=ok, ldk=256, v=ok, ldv=256, cache=(ok, ok, 8), st=ok, **over):
    return b.lib.sd_append_kv(ctypes.byref(prompts(**over)), ctypes.byref(b.sd_kv_layer(*cache)), k, ldk, v, ldv, st, None)


def attend(q=ok, ldq=1024, scale=0.1, out=8192, ldo=1024, lse=ok, ws=ok, ws_bytes=1 << 40, cache=(ok, ok, 8), st=ok, **over):
    return b.lib.sd_prompt_attention(ctypes.byref(prompts(**over)), ctypes.byref(b.sd_kv_layer(*cache)), q, ldq, f(scale), out, ldo, lse, ws,
                                     ws_bytes, st, None)


def assign(stack=ok, n_free=ok, blocks=8, B=2, W=4, table=ok, n_blocks=ok, lens=ok, new=ok, granted=None, st=ok, pool=True):
    c = b.sd_block_pool(stack, n_free, blocks)
    return b.lib.sd_assign_blocks(ctypes.byref(c) if pool else None, B, W, table, n_blocks, lens, new, granted, st, None)


@pytest.mark.parametrize("call", [prepare, append, attend])
def test_geometry(call):
    for bad in (dict(B=0), dict(N=-1), dict(Hq=0), dict(Hkv=0), dict(W=0), dict(blocks=0), dict(table=None), dict(lens=None), dict(new=None),
                dict(start=None), dict(slot=None), dict(pos=None), dict(plan=None), dict(plan=4100), dict(table=4097), dict(n_blocks=4098),
                dict(slot=4097), dict(st=None)):
        assert call(**bad) == b.SD_ERR_INVALID_ARG, bad
    for bad in (dict(D=64), dict(block=16), dict(B=8193), dict(N=(1 << 24) + 1), dict(Hq=9), dict(Hq=18), dict(blocks=(1 << 25) + 1),
                dict(Hq=1032, Hkv=129)):
        assert call(**bad) == b.SD_ERR_UNSUPPORTED, bad


def test_rows_of_heads():
    for bad in (dict(k=None), dict(v=None), dict(k=4100), dict(ldk=255), dict(ldk=252), dict(ldv=260), dict(ldv=1 << 31), dict(cache=(None, ok, 8)),
                dict(cache=(ok, 4100, 8)), dict(cache=(ok, ok, 7))):
        assert append(**bad) == b.SD_ERR_INVALID_ARG, bad
    for bad in (dict(q=None), dict(out=None), dict(out=ok), dict(q=4100), dict(ldq=1016), dict(ldq=1028), dict(ldo=1016), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(lse=4097), dict(ws=None), dict(ws=4104),
                dict(cache=(ok, ok, 9))):
        assert attend(**bad) == b.SD_ERR_INVALID_ARG, bad
    need = b.lib.sd_prompt_workspace_bytes(ctypes.byref(prompts()))
    assert need > 0 and attend(ws_bytes=need - 1) == b.SD_ERR_WORKSPACE
    # no rows: nothing is launched
    assert append(N=0, k=None, v=None) == b.SD_OK
    assert attend(N=0, q=None, out=None) == b.SD_OK


def test_tables():
    for bad in (dict(pool=False), dict(stack=None), dict(n_free=None), dict(blocks=0), dict(B=0), dict(W=0), dict(table=None), dict(n_blocks=None),
                dict(lens=None), dict(new=None), dict(st=None), dict(granted=4097), dict(stack=4098), dict(lens=4099)):
        assert assign(**bad) == b.SD_ERR_INVALID_ARG, bad
    assert assign(B=8193) == b.SD_ERR_UNSUPPORTED
    assert assign(blocks=(1 << 25) + 1) == b.SD_ERR_UNSUPPORTED


def test_caches_whose_rows_pass_32_bits():
    many = dict(Hq=64, Hkv=64, ldq=8192, ldo=8192, blocks=1 << 19, cache=(ok, ok, 1 << 19))
    assert attend(**many) == b.SD_ERR_UNSUPPORTED


def test_sizes_of_refused_geometries_are_zero():
    assert b.lib.sd_prompt_plan_bytes(ctypes.byref(prompts())) > 0
    for bad in (dict(D=64), dict(B=0), dict(Hq=9)):
        assert b.lib.sd_prompt_plan_bytes(ctypes.byref(prompts(**bad))) == 0
        assert b.lib.sd_prompt_workspace_bytes(ctypes.byref(prompts(**bad))) == 0
    assert b.lib.sd_prompt_plan_bytes(None) == 0


def test_oracle_tables_by_hand():
    table = np.array([[5, 6, 7, -1], [8, -1, -1, -1], [9, 4, -1, -1]], dtype=np.int32)
    # request 0 keeps one of three, request 1 wants three, request 2 four (of which the pool has two more: short)
    t, held, stack, n, granted = ref.assign(table, np.array([3, 1, 2], dtype=np.int32), [64, 100, 200], [0, 60, 56], [1, 2, 0, 0], 1)
    assert granted.tolist() == [1, 1, 0] and held.tolist() == [1, 3, 2] and n == 1 and stack[:1].tolist() == [1]
    assert t[1].tolist() == [8, 6, 7, -1]
    # and back
    t, held, stack, n, _ = ref.assign(t, held, [64, 64, 128], [0, 0, 0], stack, n)
    assert held.tolist() == [1, 1, 2] and n == 3 and stack[:3].tolist() == [1, 7, 6]


def test_oracle_attention_is_the_softmax_of_the_seen_keys():
    g = np.random.default_rng(0)
    table, lens, new = np.array([[2, 0], [1, 3]]), [70, 0], [3, 5]
    q, k, v = g.standard_normal((8, 4, 16)), g.standard_normal((4, 2, 64, 16)), g.standard_normal((4, 2, 64, 16))
    out, lse, _, _ = ref.attention(q, k, v, table, lens, new, 0.3)
    row = 0
    for b in range(2):
        for i in range(new[b]):
            for h in range(4):
                seen = [(table[b, t // 64], h // 2, t % 64) for t in range(lens[b] + i + 1)]
                e = np.exp([0.3 * float(q[row, h] @ k[s]) for s in seen])
                np.testing.assert_allclose(out[row, h], sum(w * v[s] for w, s in zip(e, seen)) / e.sum(), rtol=1e-12)
                np.testing.assert_allclose(lse[row, h], np.log(e.sum()), rtol=1e-12)
            row += 1
