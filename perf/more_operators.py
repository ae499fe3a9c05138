"""From requests to a filled cache: what is measured, and the operators' plain forms.

    tables     block tables sized to the requests' lengths from a pool of free blocks, the slots of the new tokens, and what the
               requests did not need given back
    append     keys and values of packed tokens into the blocks of one layer's cache
    attention  causal attention of packed new tokens, from one to a whole prompt per request, over the cache that they are in

`run` computes them in elementary torch operations, or with `own` through the library.  A block holds 64 tokens; a cache is
[blocks][KV heads][64][128] bf16, K and V each.  Request b has len[b] tokens in the cache and brings new[b]; the new tokens of all
requests stand behind one another in packed rows, those of request b from row start[b] on.
"""
import math
import random

import torch

own = False

BLOCK = 64
D = 128


def listed():
    return [
        # one step of a serving batch: each request's tree of 60 nodes needs a block now and then
        {"name": "tables_step", "op": "tables", "batch": "16*60@512..16384", "spare": 300, "lengths": 1},
        # many short requests come and go beside long ones; the pool does not suffice for all of them
        {"name": "tables_churn", "op": "tables", "batch": "700*0@0..9000 900*1..2000@0 400*1@100..16384", "spare": 13000, "lengths": 2},
        # the next token of a batch
        {"name": "append_step", "op": "append", "batch": "16*1@512..16384", "Hq": 28, "Hkv": 4, "lengths": 3},
        # prompts of a batch, ragged
        {"name": "append_prompts", "op": "append", "batch": "24*1..4096@0..300", "Hq": 28, "Hkv": 4, "lengths": 4},
        # one user's next token: latency
        {"name": "decode_one", "op": "attention", "batch": "1*1@2047", "Hq": 28, "Hkv": 4, "lengths": 5},
        # the next token of a ragged serving batch
        {"name": "decode_batch", "op": "attention", "batch": "32*1@512..16384", "Hq": 28, "Hkv": 4, "lengths": 6},
        # a piece of a long prompt beside other requests' next tokens
        {"name": "chunk_beside_decode", "op": "attention", "batch": "1*1000@7000 24*1@300..9000", "Hq": 28, "Hkv": 4, "lengths": 7},
        # a user's next question in a long conversation: few rows, many keys
        {"name": "question", "op": "attention", "batch": "1*61@16000", "Hq": 28, "Hkv": 4, "lengths": 8},
        # short and middling prompts that came in together
        {"name": "prompts_packed", "op": "attention", "batch": "16*1..2048@0", "Hq": 28, "Hkv": 4, "lengths": 9},
        # the prompts behind the batch of eight that verification is quoted on
        {"name": "prompts_4096", "op": "attention", "batch": "8*4096@0", "Hq": 28, "Hkv": 4, "lengths": 10},
        # as many KV heads as query heads, odd lengths
        {"name": "prompts_own_heads", "op": "attention", "batch": "3*100..5000@0..1000", "Hq": 12, "Hkv": 12, "lengths": 11},
        # a long multimodal context from its first token
        {"name": "prompt_long", "op": "attention", "batch": "1*32749@0", "Hq": 28, "Hkv": 4, "lengths": 12},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _spec(count, new, cached):
    span = lambda a, b: str(a) if a == b else f"{a}..{b}"
    return f"{count}*{span(*new)}@{span(*cached)}"


def draw(rng):
    op = rng.choice(("tables", "append", "attention", "attention", "attention"))
    case = {"op": op, "lengths": rng.randrange(1 << 30)}
    if op == "tables":
        B = _spread(rng, 1, 2000)
        longest = _spread(rng, 100, 16384)
        n = _spread(rng, 1, 2000)
        case["batch"] = _spec(B, (0, n), (0, longest)) + " " + _spec(_spread(rng, 1, 50), (1, 4096), (0, 0))
        case["spare"] = _spread(rng, 8, 20000)
        return case
    case["Hkv"] = rng.choice((1, 2, 4, 4, 8))
    case["Hq"] = case["Hkv"] * rng.choice((1, 2, 4, 5, 7, 7, 8))
    if op == "append":
        case["batch"] = _spec(_spread(rng, 1, 64), (1, _spread(rng, 1, 2000)), (0, _spread(rng, 1, 5000)))
        return case
    kind = rng.choice(("single", "prompts", "chunks", "mixed", "long"))
    room = 1200000 // case["Hkv"]                                     # tokens that the cache holds, about
    if kind in ("single", "mixed"):
        longest = _spread(rng, 64, 32768)
        case["batch"] = _spec(min(_spread(rng, 1, 128), max(room // longest, 1)), (1, rng.choice((1, 1, 1, 4))), (0, longest))
        if kind == "mixed":
            case["batch"] += " " + _spec(rng.randint(1, 3), (1, _spread(rng, 16, 2048)), (0, _spread(rng, 1, 8192)))
    elif kind == "prompts":
        longest = _spread(rng, 16, 4096)
        case["batch"] = _spec(min(_spread(rng, 1, 64), max(20000 // longest, 1)), (1, longest), (0, 0))
    elif kind == "chunks":
        case["batch"] = _spec(rng.randint(1, 8), (1, _spread(rng, 16, 1024)), (0, _spread(rng, 64, 16384)))
    else:
        n = _spread(rng, 2000, 16000)
        case["batch"] = _spec(1, (n, n), (0, 100))
    return case


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """[(new tokens, cached tokens)] of the case's requests, the same for every seed."""
    rng = random.Random(case["lengths"])
    out = []
    for part in case["batch"].split():
        count, rest = part.split("*")
        ends = [[int(x) for x in r.split("..")] for r in rest.split("@")]
        out += [tuple(rng.randint(e[0], e[-1]) for e in ends) for _ in range(int(count))]
    rng.shuffle(out)
    return out


def _blocks(tokens):
    return -(-tokens // BLOCK)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    lens = _lengths(case)
    B, N = len(lens), sum(n for n, _ in lens)
    ints = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")
    s = {"case": case, "lens": lens, "N": N, "new": ints([n for n, _ in lens]), "len": ints([c for _, c in lens]),
         "status": torch.zeros(1, dtype=torch.int32, device="cuda"), "handle": None}
    tables = case["op"] == "tables"
    held = [_blocks(c if tables else n + c) for n, c in lens]
    W = max(1, max(_blocks(n + c) for n, c in lens))
    pool = sum(held) + (case["spare"] if tables else 5)
    order = torch.randperm(pool, generator=g, device="cuda").int()
    table = torch.full((B, W), -1, dtype=torch.int32, device="cuda")
    there = torch.arange(W, device="cuda")[None] < ints(held)[:, None]
    table[there] = order[:sum(held)]
    s["table"], s["held"], s["num_blocks"] = table, ints(held), pool
    if tables:
        s["stack"] = torch.full((pool,), -1, dtype=torch.int32, device="cuda")
        s["stack"][:pool - sum(held)] = order[sum(held):]
        s["n_free"] = ints([pool - sum(held)])
        s["granted"], s["start"] = ints([0] * B), ints([0] * (B + 1))
        s["slot"], s["position"] = torch.full((2, N), -1, dtype=torch.int32, device="cuda")
        return s
    Hq, Hkv = case["Hq"], case["Hkv"]
    # the projection's output: q, k and v of a token side by side
    qkv = torch.randn((N, Hq + 2 * Hkv, D), generator=g, device="cuda").bfloat16()
    s["q"], s["k"], s["v"] = qkv[:, :Hq] * 1.5, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    fresh = lambda: torch.randn((pool, Hkv, BLOCK, D), generator=g, device="cuda", dtype=torch.bfloat16)
    s["k_cache"], s["v_cache"] = fresh(), fresh()
    # some keys that many queries agree on, the first one of each request among them
    s["k_cache"][:, :, ::17] *= 2.0
    if case["op"] == "attention":
        qkv[:, :Hq] = s["q"]
        s["q"] = qkv[:, :Hq]
        s["out"] = torch.zeros((N, Hq, D), dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros((N, Hq), device="cuda")
        s["scale"] = 1.0 / math.sqrt(D)
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _plain_assign(table, held, target, stack, n_free):
    """Tables that cover `target` tokens: (table, held, stack, n_free, granted)."""
    B, W = table.shape
    table, stack = table.clone(), stack.clone()
    want = (target + BLOCK - 1) // BLOCK
    grow, shrink = (want - held).clamp(min=0).long(), (held - want).clamp(min=0).long()
    free = n_free[0].long()
    P = shrink.sum()
    after = torch.cumsum(grow, dim=0)
    granted = (grow == 0) | (after <= free + P)
    grow = torch.where(granted, grow, torch.zeros_like(grow))
    after = torch.cumsum(grow, dim=0)
    Q = grow.sum()
    column = torch.arange(W, device=table.device)[None]
    # blocks that come free, request by request: those the others take first
    gives = (column >= want[:, None]) & (column < held[:, None])
    released = table[gives].long()
    takes = (column >= held[:, None]) & (column < (held + grow)[:, None])
    t = ((after - grow)[:, None] + column - held[:, None])[takes]
    from_stack = stack[(free - 1 - (t - P)).clamp(0, stack.numel() - 1)].long()
    if released.numel():
        from_stack = torch.where(t < P, released[t.clamp(0, released.numel() - 1)], from_stack)
    table[takes] = from_stack.int()
    left = torch.arange(released.numel(), device=table.device)
    keep = left >= Q
    stack[(free + P - 1 - left)[keep]] = released[keep].int()
    return table, torch.where(granted, torch.minimum(held, want) + grow, held).int(), stack, (n_free + P - Q).int(), granted.int()


def _plain_slots(table, held, length, new, N):
    start = torch.zeros(new.numel() + 1, dtype=torch.int64, device=new.device)
    start[1:] = torch.cumsum(new.long(), dim=0)
    row = torch.arange(N, device=new.device)
    b = torch.searchsorted(start, row, right=True) - 1
    position = length[b].long() + row - start[b]
    covered = (held[b].long() * BLOCK >= (length + new)[b])
    slot = table[b, (position // BLOCK).clamp(max=table.shape[1] - 1)].long() * BLOCK + position % BLOCK
    return start.int(), torch.where(covered, slot, torch.full_like(slot, -1)).int(), position.int()


def _plain_tables(s):
    table, held, stack, n_free, granted = _plain_assign(s["table"], s["held"], s["len"] + s["new"], s["stack"], s["n_free"])
    start, slot, position = _plain_slots(table, held, s["len"], s["new"], s["N"])
    table, held, stack, n_free, _ = _plain_assign(table, held, s["len"], stack, n_free)
    return {"table": table, "held": held, "stack": stack, "n_free": n_free, "granted": granted,
            "start": start, "slot": slot, "position": position}


def _plain_append(s):
    _, slot, _ = _plain_slots(s["table"], s["held"], s["len"], s["new"], s["N"])
    slot = slot.long()
    s["k_cache"][slot // BLOCK, :, slot % BLOCK] = s["k"]
    s["v_cache"][slot // BLOCK, :, slot % BLOCK] = s["v"]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attention(s):
    Hq, Hkv = s["case"]["Hq"], s["case"]["Hkv"]
    G = Hq // Hkv
    out, lse = torch.empty_like(s["out"]), torch.empty_like(s["lse"])
    row = 0
    for b, (new, cached) in enumerate(s["lens"]):
        total = cached + new
        blocks = s["table"][b, :_blocks(total)].long()
        k = s["k_cache"][blocks].transpose(0, 1).reshape(Hkv, -1, D)[:, :total].float()
        v = s["v_cache"][blocks].transpose(0, 1).reshape(Hkv, -1, D)[:, :total].float()
        key = torch.arange(total, device=k.device)
        step = max(1, (1 << 28) // (Hq * total))
        for i in range(0, new, step):
            n = min(step, new - i)
            seen = cached + i + n                                    # keys that the last of these rows sees
            q = s["q"][row + i:row + i + n].float().reshape(n, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * n, D)
            score = torch.matmul(q, k[:, :seen].transpose(1, 2)).view(Hkv, G, n, seen) * s["scale"]
            hidden = key[None, :seen] > cached + i + torch.arange(n, device=k.device)[:, None]
            score.masked_fill_(hidden, -math.inf)
            top = score.amax(dim=3, keepdim=True)
            weight = score.sub_(top).exp_()
            total_weight = weight.sum(dim=3, keepdim=True)
            o = torch.matmul(weight.view(Hkv, G * n, seen), v[:, :seen]).view(Hkv, G, n, D) / total_weight
            out[row + i:row + i + n] = o.permute(2, 0, 1, 3).reshape(n, Hq, D).to(out.dtype)
            lse[row + i:row + i + n] = (top + torch.log(total_weight))[..., 0].permute(2, 0, 1).reshape(n, Hq)
            del score, weight
        row += new
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------------------------- the library's calls
def _own(s):
    from paper_2509_18824_b200 import binding as sd
    case, status = s["case"], s["status"]
    if s["handle"] is None:
        prompts = sd.Prompts(s["N"], case.get("Hq", 1), case.get("Hkv", 1), D, s["table"], s["len"], s["new"], s["held"],
                             num_blocks=s["num_blocks"])
        if case["op"] == "tables":
            prompts.use(s["start"], s["slot"], s["position"])
            s["handle"] = (prompts, sd.BlockPool(s["num_blocks"], s["stack"], s["n_free"]), torch.zeros_like(s["new"]), torch.zeros_like(s["new"]))
        else:
            # (once for all layers of a model's step)
            sd.sd_prompt_prepare(prompts, status)
            work = torch.empty(sd.sd_prompt_workspace_bytes(prompts), dtype=torch.uint8, device="cuda")
            s["handle"] = (prompts, sd.kv_layer(s["k_cache"], s["v_cache"]), work)
    if case["op"] == "tables":
        prompts, pool, nothing, unused = s["handle"]
        sd.sd_assign_blocks(pool, s["table"], s["held"], s["len"], s["new"], s["granted"], status)
        sd.sd_prompt_prepare(prompts, status)
        sd.sd_assign_blocks(pool, s["table"], s["held"], s["len"], nothing, unused, status)
        return {"table": s["table"], "held": s["held"], "stack": s["stack"], "n_free": s["n_free"], "granted": s["granted"],
                "start": s["start"], "slot": s["slot"], "position": s["position"]}
    prompts, cache, work = s["handle"]
    if case["op"] == "append":
        sd.sd_append_kv(prompts, cache, s["k"], s["v"], status)
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    sd.sd_prompt_attention(prompts, cache, s["q"], s["scale"], s["out"], s["lse"], work, status)
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    return {"tables": _plain_tables, "append": _plain_append, "attention": _plain_attention}[state["case"]["op"]](state)


def work(case):
    lens = _lengths(case)
    N = sum(n for n, _ in lens)
    if case["op"] == "tables":
        moved = sum(_blocks(n + c) - _blocks(c) for n, c in lens)
        # lengths and counts of both calls, the entries that move and move back, the packed rows' arrays
        return {"bytes": len(lens) * 28 + 16 * min(moved, case["spare"]) + 8 * N, "flops": 4 * N}
    if case["op"] == "append":
        return {"bytes": N * (8 * case["Hkv"] * D + 4), "flops": 0}
    Hq, Hkv = case["Hq"], case["Hkv"]
    seen = sum(n * c + n * (n + 1) // 2 for n, c in lens)
    keys = sum(c + n for n, c in lens if n)
    return {"bytes": N * Hq * (4 * D + 4) + keys * Hkv * D * 4, "flops": 4 * D * Hq * seen}


# ---------------------------------------------------------------------------------------------- in 64 bits, from the definition
def exact(case, seed):
    """The attention of each head over the cache, row after row of queries in 64 bits.  (Tables and copies have no rounding.)"""
    lens = _lengths(case)
    if case["op"] != "attention" or case["Hq"] * sum(n * (c + n) for n, c in lens) > 1 << 34:
        return None
    s = prepare(case, seed)
    Hq, Hkv = case["Hq"], case["Hkv"]
    out, lse = [], []
    first = 0
    for b, (new, cached) in enumerate(lens):
        t = torch.arange(cached + new, device="cuda")
        block, offset = s["table"][b].long()[t // BLOCK], t % BLOCK
        here = torch.empty((new, Hq, D), dtype=torch.float64, device="cuda")
        here_lse = torch.empty((new, Hq), dtype=torch.float64, device="cuda")
        step = max(1, (1 << 26) // (cached + new))
        for h in range(Hq):
            k, v = (s[c][block, h * Hkv // Hq, offset].double() for c in ("k_cache", "v_cache"))
            for i in range(0, new, step):
                rows = torch.arange(i, min(i + step, new), device="cuda")
                z = (s["q"][first + rows, h].double() @ k.T) / math.sqrt(D)
                z = torch.where(t[None] <= cached + rows[:, None], z, torch.full((), -math.inf, dtype=torch.float64, device="cuda"))
                here_lse[rows, h] = torch.logsumexp(z, dim=1)
                here[rows, h] = torch.softmax(z, dim=1) @ v
        out.append(here)
        lse.append(here_lse)
        first += new
    return {"out": torch.cat(out), "lse": torch.cat(lse)}
