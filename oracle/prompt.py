"""From requests to a filled cache, in plain Python and 64 bits: block tables from lengths, slots of packed tokens, K/V into their
slots, causal attention over the cache.  Written from the definitions in include/sdverify.h; shares no code with the library."""
import numpy as np

BLOCK = 64


def assign(table, n_blocks, lens, n_new, stack, n_free, short_of=None):
    """(table, n_blocks, stack, n_free, granted) behind one call; stack: list whose first n_free entries count (the top is the last)."""
    table, n_blocks, stack = table.copy(), n_blocks.copy(), list(stack)
    B = len(lens)
    want = [-(-(int(lens[b]) + int(n_new[b])) // BLOCK) for b in range(B)]
    free = stack[:n_free]
    returned = []                                            # in the order of the requests and of their tables
    for b in range(B):
        returned += [int(x) for x in table[b, want[b]:n_blocks[b]]]
    free += returned[::-1]                                   # the first one given back comes out first
    granted = np.ones(B, dtype=np.int32)
    short = False
    held = [min(int(n_blocks[b]), want[b]) for b in range(B)]
    for b in range(B):
        grow = want[b] - held[b]
        if grow > 0 and (short or grow > len(free)):
            short = True
            granted[b] = 0
            continue
        for j in range(grow):
            table[b, held[b] + j] = free.pop()
        held[b] += grow
    after = len(free)
    return table, np.array(held, dtype=np.int32), np.array(free + [int(x) for x in stack[after:]], dtype=np.int32), after, granted


def slots(table, n_blocks, lens, n_new, N):
    start = np.concatenate([[0], np.cumsum(n_new)]).astype(np.int32)
    slot, position = np.full(N, -1, dtype=np.int32), np.zeros(N, dtype=np.int32)
    for b in range(len(lens)):
        for i in range(int(n_new[b])):
            t = int(lens[b]) + i
            position[start[b] + i] = t
            if int(n_blocks[b]) * BLOCK >= int(lens[b]) + int(n_new[b]):
                slot[start[b] + i] = table[b, t // BLOCK] * BLOCK + t % BLOCK
    return start, slot, position


def attention(q, k_cache, v_cache, table, lens, n_new, scale):
    """q [N,Hq,D], caches [blocks,Hkv,64,D] (float64) -> out, lse, and two sizes that rounding is measured by: sum of weight x |V| of each
    output, and the largest scale x sum |q||k| of each row."""
    N, Hq, D = q.shape
    Hkv = k_cache.shape[1]
    out, lse = np.zeros((N, Hq, D)), np.zeros((N, Hq))
    spread, size = np.zeros((N, Hq, D)), np.zeros((N, Hq))
    row = 0
    for b in range(len(lens)):
        n, c = int(n_new[b]), int(lens[b])
        t = np.arange(c + n)
        for h in range(Hq):
            k = k_cache[table[b, t // BLOCK], h * Hkv // Hq, t % BLOCK]
            v = v_cache[table[b, t // BLOCK], h * Hkv // Hq, t % BLOCK]
            if n == 0:
                continue
            z = q[row:row + n, h] @ k.T * scale
            z[t[None] > c + np.arange(n)[:, None]] = -np.inf
            top = z.max(axis=1, keepdims=True)
            w = np.exp(z - top)
            total = w.sum(axis=1, keepdims=True)
            w /= total
            out[row:row + n, h] = w @ v
            spread[row:row + n, h] = w @ np.abs(v)
            lse[row:row + n, h] = (top + np.log(total))[:, 0]
            size[row:row + n, h] = (np.abs(q[row:row + n, h]) @ np.abs(k).T).max(axis=1) * scale
        row += n
    return out, lse, spread, size
