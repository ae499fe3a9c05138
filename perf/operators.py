"""Operators on rows of logits: what is measured, and their plain forms.

    top      the K largest logits of a row with the row's log-sum-exp: a teacher's rows for distillation, a draft
             node's candidates for the tree's next level
    sample   tokens drawn from a row at a temperature, behind top-k, top-p and min-p, from given uniform numbers: the
             draft's tokens, with their probabilities and (optionally) the whole distribution that the acceptance rules read
    filter   the same temperature and filters on the target's logits, for verification against a filtered target
    distill  KL from a teacher's top logits plus cross-entropy (the draft's training loss), and its gradient

`run` computes them in elementary torch operations, or with `own` through the library.  Rows are ordered by (logit
descending, index ascending); masses, their sums and the borders that they are compared with are held in 64 bits: a
token next to a border would otherwise fall to either side.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
#: sampling parameters of a batch: what its rows ask for
MODES = ("usual", "mixed", "temperature", "top_p", "min_p")


def listed():
    return [
        # one user's next token from the vocabulary of the 7B-shaped workloads: latency
        {"name": "sample_one_row", "op": "sample", "M": 1, "V": 152064, "type": "f32", "N": 1, "mode": "usual", "probs": False},
        # a serving batch whose requests ask for different filters, some of them greedy
        {"name": "sample_batch", "op": "sample", "M": 64, "V": 152064, "type": "f32", "N": 1, "mode": "mixed", "probs": False},
        # a draft level: four children drawn per node, the distributions kept for the acceptance rule; odd vocabulary
        {"name": "sample_draft_level", "op": "sample", "M": 80, "V": 32003, "type": "bf16", "N": 4, "mode": "top_p", "probs": True},
        # rollouts at a temperature alone
        {"name": "sample_temperature", "op": "sample", "M": 256, "V": 152064, "type": "f32", "N": 1, "mode": "temperature", "probs": False},
        # root and ten drafts of one sequence
        {"name": "filter_chain", "op": "filter", "M": 11, "V": 152064, "type": "f32", "mode": "top_p"},
        # eight trees of 60 nodes
        {"name": "filter_trees", "op": "filter", "M": 480, "V": 152064, "type": "f32", "mode": "mixed"},
        # ten candidates of each of ten frontier nodes, eight sequences
        {"name": "top_expand", "op": "top", "M": 80, "V": 152064, "type": "f32", "K": 10},
        # a teacher's rows of a training batch
        {"name": "top_teacher", "op": "top", "M": 4096, "V": 152064, "type": "bf16", "K": 64},
        # a small vocabulary in 32 bits, at a temperature, without the rest of the teacher's mass
        {"name": "distill_small", "op": "distill", "M": 61, "V": 4099, "type": "f32", "K": 10, "form": "both", "tail": False, "inv_temp": 0.5},
        # the training step's loss and gradient in one call
        {"name": "distill_train", "op": "distill", "M": 4096, "V": 152064, "type": "bf16", "K": 64, "form": "both", "tail": True, "inv_temp": 1.0},
        # evaluation: the loss alone
        {"name": "distill_loss", "op": "distill", "M": 1000, "V": 152064, "type": "bf16", "K": 64, "form": "loss", "tail": True, "inv_temp": 1.0},
        # loss first, the gradient in a call of its own when the rows' weights are known
        {"name": "distill_two_calls", "op": "distill", "M": 512, "V": 50001, "type": "f32", "K": 128, "form": "two", "tail": True, "inv_temp": 1.25},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("sample", "sample", "filter", "top", "distill", "distill"))
    V = 152064 if rng.random() < 0.3 else _spread(rng, 300, 200000)
    case = {"op": op, "V": V, "type": rng.choice(("f32", "bf16"))}
    if op in ("sample", "filter"):
        case["M"] = _spread(rng, 1, min(480, 73000000 // V))
        case["mode"] = rng.choice(MODES)
        if op == "sample":
            case["N"] = rng.choice((1, 1, 2, 4, 10))
            case["probs"] = rng.random() < 0.4
    else:
        case["M"] = _spread(rng, 1, min(8192, 300000000 // V))
        case["K"] = min(_spread(rng, 4, 500), V // 4)
        if op == "distill":
            case["form"] = rng.choice(("both", "both", "loss", "two"))
            case["tail"] = rng.random() < 0.7
            case["inv_temp"] = rng.choice((1.0, 1.0, 0.5, 1.25))
    return case


# ---------------------------------------------------------------------------------------------- inputs
def _logits(g, M, V, dtype):
    """Rows as language models give them: a broad bulk, and some dozens of tokens above it by more or less."""
    x = torch.randn((M, V), generator=g, device="cuda") * 2.0
    n = min(64, V)
    part = V // n                                                            # the tokens are distinct: one in each n-th of the vocabulary
    at = torch.arange(n, device="cuda") * part + torch.rand((M, n), generator=g, device="cuda").mul_(part).long().clamp_(max=part - 1)
    rank = torch.argsort(torch.rand((M, n), generator=g, device="cuda"), dim=1)
    height = 16.0 * torch.rand((M, 1), generator=g, device="cuda") - 1.5 * torch.log1p(rank.float())
    x.scatter_(1, at, height.clamp(min=0.0) + torch.rand((M, n), generator=g, device="cuda"))
    return x.to(dtype)


def _choice(g, values, M):
    v = torch.tensor(values, device="cuda")
    return v[torch.randint(0, len(values), (M,), generator=g, device="cuda")]


def _params(g, mode, M):
    """inv_temp, top_k, top_p, min_p of every row, None where nobody in the batch uses one."""
    it = 0.7 + torch.rand(M, generator=g, device="cuda")
    if mode == "usual":
        return it, _choice(g, [40, 50], M).int(), _choice(g, [0.9, 0.95], M), None
    if mode == "temperature":
        return it, None, None, None
    if mode == "top_p":
        return it, None, 0.8 + 0.19 * torch.rand(M, generator=g, device="cuda"), None
    if mode == "min_p":
        return it, None, None, _choice(g, [0.02, 0.05, 0.1], M)
    it = torch.where(torch.rand(M, generator=g, device="cuda") < 0.1, torch.full_like(it, math.inf), it)
    return it, _choice(g, [0, 0, 20, 50, 200, 5000], M).int(), _choice(g, [1.0, 0.8, 0.9, 0.95, 0.99], M), _choice(g, [0.0, 0.0, 0.02, 0.1], M)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    M, V, op = case["M"], case["V"], case["op"]
    dtype = TYPES[case["type"]]
    empty = lambda shape, t=torch.float32: torch.empty(shape, dtype=t, device="cuda")
    s = {"case": case, "x": _logits(g, M, V, dtype), "status": torch.zeros(1, dtype=torch.int32, device="cuda"), "handle": None}
    if op in ("sample", "filter"):
        s["params"] = _params(g, case["mode"], M)
        s["lse"] = empty((M,))
        if op == "sample":
            s["u"] = torch.rand((M, case["N"]), generator=g, device="cuda")
            s["tokens"], s["prob"] = empty((M, case["N"]), torch.int32), empty((M, case["N"]))
            s["probs"] = empty((M, V)) if case["probs"] else None
        else:
            s["out"], s["kept"] = empty((M, V)), empty((M,), torch.int32)
    elif op == "top":
        s["values"], s["index"], s["lse"] = empty((M, case["K"])), empty((M, case["K"]), torch.int32), empty((M,))
    else:
        K, it = case["K"], case["inv_temp"]
        # the teacher agrees with the student about the bulk and not quite about the top
        teacher = 0.5 * torch.randn((M, V), generator=g, device="cuda")
        teacher += s["x"]
        s["t_val"], index = torch.topk(teacher, K, dim=1)
        s["t_idx"] = index.int()
        s["t_lse"] = torch.logsumexp(teacher.mul_(it), dim=1) if case["tail"] else None
        del teacher, index
        # one entry in twenty lies outside the draft's vocabulary, some labels too
        s["t_idx"][torch.rand((M, K), generator=g, device="cuda") < 0.05] = -1
        s["label"] = torch.randint(0, V, (M,), generator=g, device="cuda").int()
        s["label"][torch.rand(M, generator=g, device="cuda") < 0.3] = -1
        s["dloss"] = torch.rand(M, generator=g, device="cuda") / M * 64
        s["kl"], s["ce"], s["stats"] = empty((M,)), empty((M,)), empty((M, 4))
        s["grad"] = empty((M, V), dtype) if case["form"] != "loss" else None
    return s


# ---------------------------------------------------------------------------------------------- plain forms
def _kept(x, params):
    """x [M, V] f32 -> the rows in order (values, indices), their masses relative to the largest (f64), and which of them stay."""
    it, k, p, mp = params
    M, V = x.shape
    greedy = torch.isinf(it)[:, None]
    scale = torch.where(greedy[:, 0], torch.ones_like(it), it).double()[:, None]
    value, index = torch.sort(x, dim=1, descending=True, stable=True)
    mass = torch.exp((value.double() - value[:, :1].double()) * scale)
    rank = torch.arange(V, device=x.device)[None]
    stay = ~greedy | (rank < 1)
    if k is not None:
        k = k[:, None]
        stay = stay & ((k < 1) | (rank < k))
    if p is not None:
        m = torch.where(stay, mass, torch.zeros_like(mass))
        c = torch.cumsum(m, dim=1)
        p = p.double()[:, None]
        stay = stay & ((p >= 1) | (c - m < p * c[:, -1:]) | (rank < 1))
    if mp is not None:
        mp = mp.double()[:, None]
        stay = stay & ((mp <= 0) | (mass >= mp.clamp(max=1.0)))
    return value, index, mass, stay, scale


def _plain_sample(s):
    x = s["x"].float()
    value, index, mass, stay, scale = _kept(x, s["params"])
    w = torch.zeros_like(mass).scatter_(1, index, mass * stay)               # in vocabulary order
    c = torch.cumsum(w, dim=1)
    total = c[:, -1:]
    tokens = torch.searchsorted(c, s["u"].double() * total, right=True).clamp(max=x.shape[1] - 1)
    out = {"tokens": tokens.int(), "prob": (torch.gather(w, 1, tokens) / total).float(),
           "lse": (value[:, 0].double() * scale[:, 0] + torch.log(total[:, 0])).float()}
    if s["case"]["probs"]:
        out["probs"] = (w / total).float()
    return out


def _plain_filter(s):
    x = s["x"].float()
    value, index, mass, stay, scale = _kept(x, s["params"])
    total = (mass * stay).sum(dim=1)
    scaled = torch.where(stay, (value.double() * scale).float(), torch.full_like(value, -math.inf))
    return {"out": torch.empty_like(x).scatter_(1, index, scaled), "kept": stay.sum(dim=1).int(),
            "lse": (value[:, 0].double() * scale[:, 0] + torch.log(total)).float()}


def _plain_top(s):
    x = s["x"].float()
    value, index = torch.sort(x, dim=1, descending=True, stable=True)
    top = value[:, :1]
    lse = top[:, 0] + torch.log(torch.exp(x - top).sum(dim=1))
    K = s["case"]["K"]
    return {"values": value[:, :K].contiguous(), "index": index[:, :K].int(), "lse": lse}


def _plain_distill(s):
    case = s["case"]
    it, K = case["inv_temp"], case["K"]
    z = s["x"].float()
    M, V = z.shape
    # the teacher's distribution over its listed tokens (and the rest)
    there = s["t_idx"] >= 0
    at = s["t_idx"].clamp(min=0).long()
    t = torch.where(there, s["t_val"].double() * it, torch.full((), -math.inf, dtype=torch.float64, device=z.device))
    if case["tail"]:
        p = torch.exp(t - s["t_lse"].double()[:, None])
        p_rest = (1.0 - p.sum(dim=1)).clamp(min=0.0)
        log_p = t - s["t_lse"].double()[:, None]
    else:
        high = t.amax(dim=1, keepdim=True).clamp(min=-1e300)
        e = torch.exp(t - high)
        total = e.sum(dim=1, keepdim=True)
        p = e / total.clamp(min=1e-300)
        log_p = t - high - torch.log(total.clamp(min=1e-300))
    # the student's
    zt = z * it
    top = zt.amax(dim=1, keepdim=True)
    e = torch.exp(zt - top)
    total = e.sum(dim=1, keepdim=True, dtype=torch.float64)
    listed_mask = torch.zeros((M, V + 1), dtype=torch.bool, device=z.device)
    listed_mask.scatter_(1, torch.where(there, at, torch.full_like(at, V)), True)
    listed_mask = listed_mask[:, :V]
    log_s = torch.gather(z, 1, at).double() * it - top.double() - torch.log(total)
    kl = torch.where(there, p * (log_p - log_s), torch.zeros_like(p)).sum(dim=1)
    dist = torch.zeros((M, V + 1), device=z.device)
    dist.scatter_add_(1, torch.where(there, at, torch.full_like(at, V)), p.float())
    dist = dist[:, :V]
    soft = e / total.float()
    if case["tail"]:
        s_rest = torch.where(listed_mask, torch.zeros_like(e), e).sum(dim=1, dtype=torch.float64) / total[:, 0]
        has = (p_rest > 0) & (s_rest > 0)
        kl = kl + torch.where(has, p_rest * (torch.log(p_rest.clamp(min=1e-300)) - torch.log(s_rest.clamp(min=1e-300))), torch.zeros_like(kl))
        ratio = torch.where(has, p_rest / s_rest.clamp(min=1e-300), torch.zeros_like(p_rest)).float()
    label, has_label = s["label"].clamp(min=0).long()[:, None], s["label"] >= 0
    top1 = z.amax(dim=1, keepdim=True)
    e1 = torch.exp(z - top1)
    total1 = e1.sum(dim=1, keepdim=True)
    ce = torch.where(has_label, (torch.log(total1) + top1 - torch.gather(z, 1, label))[:, 0], torch.zeros(M, device=z.device))
    out = {"kl": kl.float(), "ce": ce}
    if case["form"] != "loss":
        d_kl = soft - dist
        if case["tail"]:
            d_kl = torch.where(listed_mask, d_kl, soft * (1.0 - ratio)[:, None])
        else:
            d_kl = d_kl * there.any(dim=1)[:, None]
        d_ce = e1 / total1
        d_ce.scatter_add_(1, label, torch.full_like(top1, -1.0))
        d_ce = d_ce * has_label[:, None]
        out["grad"] = ((it * d_kl + 0.1 * d_ce) * s["dloss"][:, None]).to(s["x"].dtype)
    return out


# ---------------------------------------------------------------------------------------------- the library's calls
def _own(s):
    from paper_2509_18824_b200 import binding as sd
    case = s["case"]
    op, status = case["op"], s["status"]
    if op == "top":
        sd.sd_top_logits(s["x"], 1.0, s["values"], s["index"], s["lse"], status)
        return {"values": s["values"], "index": s["index"], "lse": s["lse"]}
    if op in ("sample", "filter") and s["handle"] is None:
        s["handle"] = sd.Sampling(*s["params"])
    if op == "sample":
        sd.sd_sample_logits(s["x"], s["handle"], s["u"], s["tokens"], s["prob"], s["probs"], s["lse"], status)
        out = {"tokens": s["tokens"], "prob": s["prob"], "lse": s["lse"]}
        if case["probs"]:
            out["probs"] = s["probs"]
        return out
    if op == "filter":
        sd.sd_filter_logits(s["x"], s["handle"], s["out"], s["lse"], s["kept"], status)
        return {"out": s["out"], "kept": s["kept"], "lse": s["lse"]}
    teacher = (s["t_val"], s["t_idx"], s["t_lse"], s["label"], case["inv_temp"], 1.0, 0.1)
    if case["form"] == "both":
        sd.sd_distill_loss(s["x"], *teacher, s["kl"], s["ce"], s["stats"], s["dloss"], s["grad"], status)
    else:
        sd.sd_distill_loss(s["x"], *teacher, s["kl"], s["ce"], s["stats"], None, None, status)
    if case["form"] == "two":
        sd.sd_distill_grad(s["x"], *teacher, s["stats"], s["dloss"], s["grad"], status)
    out = {"kl": s["kl"], "ce": s["ce"]}
    if case["form"] != "loss":
        out["grad"] = s["grad"]
    return out


def run(state):
    if own:
        return _own(state)
    return {"sample": _plain_sample, "filter": _plain_filter, "top": _plain_top, "distill": _plain_distill}[state["case"]["op"]](state)


def work(case):
    M, V = case["M"], case["V"]
    es = 4 if case["type"] == "f32" else 2
    read = M * V * es
    if case["op"] == "sample":
        return {"bytes": read + M * (16 + 4 + 12 * case["N"]) + (4 * M * V if case["probs"] else 0), "flops": 3 * M * V}
    if case["op"] == "filter":
        return {"bytes": read + 4 * M * V + M * 24, "flops": 3 * M * V}
    K = case["K"]
    if case["op"] == "top":
        return {"bytes": read + M * (8 * K + 4), "flops": 4 * M * V}
    teacher = M * (8 * K + 4 + 4 + 4 + 8)
    if case["form"] == "loss":
        return {"bytes": read + teacher, "flops": 4 * M * V}
    # (two calls: the logits are needed before the weights are known, and again behind them)
    return {"bytes": (2 if case["form"] == "two" else 1) * read + M * V * es + teacher, "flops": 8 * M * V}


# ---------------------------------------------------------------------------------------------- in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    return {"sample": _exact_rows, "filter": _exact_rows, "top": _exact_top, "distill": _exact_distill}[case["op"]](case, s)


def _exact_rows(case, s):
    """One row after the other on the host."""
    M, V = case["M"], case["V"]
    it, k, p, mp = (None if t is None else t.cpu().numpy().astype(np.float64) for t in s["params"])
    sample = case["op"] == "sample"
    lse = np.empty(M)
    prob = np.empty((M, case["N"])) if sample else None
    probs = np.zeros((M, V)) if sample and case["probs"] else None
    out = np.full((M, V), -np.inf) if not sample else None
    for r in range(M):
        x = s["x"][r].double().cpu().numpy()
        z = x * (1.0 if np.isinf(it[r]) else it[r])
        high = z.max()
        stay = np.ones(V, dtype=bool)
        limit = 1 if np.isinf(it[r]) else (int(k[r]) if k is not None and k[r] >= 1 else V)
        q = p[r] if p is not None else 1.0
        if limit < V or q < 1.0:
            order = np.argsort(-x, kind="stable")[:limit]
            if q < 1.0:
                c = np.cumsum(np.exp(z[order] - high))
                order = order[:1 + np.searchsorted(c, q * c[-1], side="left")]
            stay[:] = False
            stay[order] = True
        if mp is not None and mp[r] > 0:
            stay &= z - high >= math.log(mp[r]) - 1e-15
        e = np.where(stay, np.exp(z - high), 0.0)
        total = e.sum()
        lse[r] = high + math.log(total)
        if sample:
            c = np.cumsum(e)
            u = s["u"][r].double().cpu().numpy()
            prob[r] = e[np.minimum(np.searchsorted(c, u * c[-1], side="right"), V - 1)] / total
            if probs is not None:
                probs[r] = e / total
        else:
            out[r, stay] = z[stay]
    if not sample:
        return {"out": out, "kept": None, "lse": lse}
    got = {"tokens": None, "prob": prob, "lse": lse}
    if probs is not None:
        got["probs"] = probs
    return got


def _exact_top(case, s):
    x, rows = s["x"], max(1, 40000000 // case["V"])
    values, lse = [], []
    for r in range(0, case["M"], rows):
        parts = x[r:r + rows].double()
        values.append(torch.topk(parts, case["K"], dim=1).values)
        lse.append(torch.logsumexp(parts, dim=1))
    return {"values": torch.cat(values), "index": None, "lse": torch.cat(lse)}


def _exact_distill(case, s):
    """The loss as it is defined, and its gradient by differentiation."""
    it, M, V = case["inv_temp"], case["M"], case["V"]
    rows = max(1, 20000000 // V)
    kl, ce, grad = [], [], []
    for r in range(0, M, rows):
        cut = slice(r, min(M, r + rows))
        z = s["x"][cut].double().requires_grad_(True)
        with torch.enable_grad():
            log_s = torch.log_softmax(z * it, dim=1)
            there = s["t_idx"][cut] >= 0
            at = s["t_idx"][cut].clamp(min=0).long()
            t = (s["t_val"][cut].double() * it).masked_fill(~there, -math.inf)
            if case["tail"]:
                t = t - s["t_lse"][cut].double()[:, None]
            else:
                t = torch.where(there.any(dim=1, keepdim=True), torch.log_softmax(t, dim=1), t)
            p = torch.exp(t)
            a = torch.where(there, p * (torch.where(there, t, torch.zeros_like(t)) - torch.gather(log_s, 1, at)), torch.zeros_like(p)).sum(dim=1)
            if case["tail"]:
                rest = (1.0 - p.sum(dim=1)).clamp(min=0.0)
                hidden = torch.zeros((z.shape[0], V + 1), dtype=torch.bool, device=z.device)
                hidden.scatter_(1, torch.where(there, at, torch.full_like(at, V)), True)
                log_rest = torch.logsumexp(log_s.masked_fill(hidden[:, :V], -math.inf), dim=1)
                a = a + torch.where(rest > 0, rest * (torch.log(rest.clamp(min=1e-300)) - log_rest), torch.zeros_like(rest))
            label = s["label"][cut].long()
            b = torch.where(label >= 0, -torch.gather(torch.log_softmax(z, dim=1), 1, label.clamp(min=0)[:, None])[:, 0], torch.zeros_like(a))
            if case["form"] != "loss":
                ((a + 0.1 * b) * s["dloss"][cut].double()).sum().backward()
                grad.append(z.grad)
        kl.append(a.detach())
        ce.append(b.detach())
    out = {"kl": torch.cat(kl), "ce": torch.cat(ce)}
    if grad:
        out["grad"] = torch.cat(grad)
    return out
