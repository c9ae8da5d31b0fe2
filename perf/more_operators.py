"""Operators that let the pages of full-precision keys and values be shared and be thinned out, as cases.

Requests that start from one text (a system prompt, a document with many questions) hold the same first pages in their
block tables; the attention of their new tokens reads those keys once for all of them.  And a request that may not grow
keeps the tokens that attention has used: attention adds up every cached token's weight, from time to time the tokens to
keep are selected by it (the first ones pinned, the last ones kept, the rest by weight), and their rows move to the front
of the request's pages so that the pages behind them are free again.

With `own` false, `run` computes each operator in elementary torch operations; with `own` true it calls the framework.
Head counts, lengths and types are those of the repository's workloads (32 query heads over 8 or 32, contexts of 512 to
32768, head dimension 128).
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
DEV = "cuda:0"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
SCALE = math.log2(math.e) / math.sqrt(D)


# ---------------------------------------------------------------- cases
def listed():
    return [
        # eight conversations behind a system prompt of about a thousand tokens, just begun: latency
        dict(name="shared step 8 on 1000", op="shared", dtype="bf16", groups=1, per_lo=8, per_hi=8, hq=32, hkv=8, page=16,
             sh_lo=1000, sh_hi=1000, own_lo=1, own_hi=64, new_lo=1, new_hi=1, scored=False, heads_first=False, mix=1),
        # a document of workload 3's length and many questions about it
        dict(name="shared 64 on 8192", op="shared", dtype="fp16", groups=1, per_lo=64, per_hi=64, hq=32, hkv=8, page=64,
             sh_lo=8192, sh_hi=8192, own_lo=16, own_hi=1024, new_lo=1, new_hi=1, scored=False, heads_first=False, mix=2),
        # several prompts in one batch, one query head per key head (workload 4's heads)
        dict(name="shared 4 prompts mha", op="shared", dtype="fp16", groups=4, per_lo=8, per_hi=16, hq=32, hkv=32, page=64,
             sh_lo=2000, sh_hi=4096, own_lo=1, own_hi=512, new_lo=1, new_hi=1, scored=False, heads_first=True, mix=3),
        # workload 5's context under a large batch whose own tokens are weighed for eviction
        dict(name="shared 128 on 30000 scored", op="shared", dtype="bf16", groups=1, per_lo=128, per_hi=128, hq=32, hkv=8,
             page=64, sh_lo=30001, sh_hi=30001, own_lo=1, own_hi=2048, new_lo=1, new_hi=1, scored=True, heads_first=False,
             mix=4),
        # few short requests with weights: latency
        dict(name="scored decode 4x512", op="scored", dtype="bf16", req=4, hq=32, hkv=8, page=16, past_lo=200, past_hi=512,
             new_lo=1, new_hi=1, window=0, sinks=0, pin=4, heads_first=False, mix=5),
        # workload 4's heads: the most bytes
        dict(name="scored decode mha 32x4096", op="scored", dtype="fp16", req=32, hq=32, hkv=32, page=64, past_lo=2048,
             past_hi=4096, new_lo=1, new_hi=1, window=0, sinks=0, pin=0, heads_first=False, mix=6),
        # a chunk of a long prompt: the weights of its rows over workload 5's context
        dict(name="scored chunk 2048 at 16000", op="scored", dtype="bf16", req=1, hq=32, hkv=8, page=64, past_lo=16000,
             past_hi=16000, new_lo=2048, new_hi=2048, window=0, sinks=0, pin=0, heads_first=True, mix=7),
        # a step of ragged chunks under workload 3's window
        dict(name="scored window chunks 8", op="scored", dtype="fp16", req=8, hq=32, hkv=8, page=16, past_lo=500, past_hi=8192,
             new_lo=50, new_hi=700, window=4096, sinks=4, pin=0, heads_first=False, mix=8),
        # a few short requests over their budget: latency
        dict(name="select 4x512", op="select", req=4, hkv=8, page=16, n_lo=300, n_hi=512, keep=256, recent=64, pin=4, mix=9),
        # long prompts to an eighth
        dict(name="select 64x16384", op="select", req=64, hkv=8, page=64, n_lo=8192, n_hi=16384, keep=2048, recent=256, pin=4,
             mix=10),
        # running requests, one page over their budget each
        dict(name="compact 4 by a page", op="compact", dtype="fp16", req=4, hkv=8, page=64, n_lo=577, n_hi=640, keep=512,
             recent=64, pin=4, heads_first=False, mix=11),
        # prompts of workload 3 to a quarter
        dict(name="compact 16x8192", op="compact", dtype="bf16", req=16, hkv=8, page=16, n_lo=5000, n_hi=8192, keep=2048,
             recent=128, pin=16, heads_first=False, mix=12),
    ]


def _log(rng, lo, hi):
    """A whole number of lo .. hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(1, lo) - 0.499), math.log(hi + 0.499)))))))


def _range(rng, lo, hi):
    a, b = sorted((_log(rng, lo, hi), _log(rng, lo, hi)))
    return a, b


def draw(rng):
    while True:
        op = rng.choice(["shared", "shared", "scored", "scored", "select", "compact"])
        mix = rng.randrange(1 << 30)
        page = rng.choice([16, 32, 64, 128, 256])
        dtype = rng.choice(["fp16", "bf16"])
        heads_first = rng.random() < 0.5
        hkv = rng.choice([1, 2, 4, 8, 8, 32])
        group = rng.choice([1, 2, 3, 4, 4, 5, 8]) if hkv < 32 else 1
        if op in ("select", "compact"):
            lo, hi = _range(rng, 64, 16384)
            keep = _log(rng, 32, max(33, hi // 2))
            case = dict(op=op, req=_log(rng, 1, 64), hkv=hkv, page=page, n_lo=lo, n_hi=hi, keep=keep,
                        recent=rng.choice([0, 1, keep // 8, keep // 2]), pin=rng.choice([0, 1, 4, 16]), mix=mix)
            if op == "compact":
                case.update(dtype=dtype, heads_first=heads_first)
            if case["req"] * hkv * hi > (8 << 20 if op == "select" else 1 << 20) or case["recent"] + case["pin"] > keep:
                continue
            if max(_lengths(case)) <= keep:      # (nobody is over the budget)
                continue
            return case
        if op == "shared":
            per = _range(rng, 2, 128)
            sh, own_ = _range(rng, 64, 32768), _range(rng, 1, 2048)
            new = (1, 1) if group > 4 else _range(rng, 1, 2)
            case = dict(op=op, dtype=dtype, groups=_log(rng, 1, 8), per_lo=per[0], per_hi=per[1], hq=hkv * group, hkv=hkv,
                        page=page, sh_lo=sh[0], sh_hi=sh[1], own_lo=own_[0], own_hi=own_[1], new_lo=new[0], new_hi=new[1],
                        scored=rng.random() < 0.3, heads_first=heads_first, mix=mix)
            req, s = case["groups"] * per[1], own_[1] + new[1]
            if req > 256 or req * hkv * s > 4e6 or case["groups"] * hkv * sh[1] > 1 << 20 \
                    or req * case["hq"] * new[1] * (sh[1] + s) > 4e8:
                continue
        else:
            single = rng.random() < 0.5
            past = _range(rng, 1, 16384)
            new = (1, 1) if single else _range(rng, 1, 2048)
            window, sinks = rng.choice([(0, 0), (0, 0), (0, 0), (_log(rng, 16, 8192), rng.choice([0, 1, 4, 100]))])
            case = dict(op=op, dtype=dtype, req=_log(rng, 1, 64 if single else 16), hq=hkv * group, hkv=hkv, page=page,
                        past_lo=past[0], past_hi=past[1], new_lo=new[0], new_hi=new[1], window=window, sinks=sinks,
                        pin=rng.choice([0, 0, 4, 100]), heads_first=heads_first, mix=mix)
            s = past[1] + new[1]
            if case["req"] * case["hq"] * new[1] * s > 1.1e9 or case["req"] * hkv * s > 4e6:
                continue
        w = work(case)
        if w["bytes"] <= 1.4e9 and w["flops"] <= 8e11:
            return case


# ---------------------------------------------------------------- lengths, the case's own whatever the seed
def _one(r, lo, hi):
    return lo if lo == hi else _log(r, lo, hi) if hi > 16 * max(1, lo) else r.randint(lo, hi)


def _requests(case):
    """(tokens cached before the step, new tokens, shared tokens) of each request, and where the groups begin."""
    r = random.Random(case["mix"])
    past, new, shared, starts = [], [], [], [0]
    if case["op"] == "shared":
        for _ in range(case["groups"]):
            per, sh = _one(r, case["per_lo"], case["per_hi"]), _one(r, case["sh_lo"], case["sh_hi"])
            past += [sh + _one(r, case["own_lo"], case["own_hi"]) - 1 for _ in range(per)]
            shared += [sh] * per
            starts.append(starts[-1] + per)
    else:
        past = [_one(r, case["past_lo"], case["past_hi"]) for _ in range(case["req"])]
        shared = [0] * case["req"]
    new = [_one(r, case["new_lo"], case["new_hi"]) for _ in past]
    return past, new, shared, starts


def _lengths(case):
    r = random.Random(case["mix"])
    return [_one(r, case["n_lo"], case["n_hi"]) for _ in range(case["req"])]


def _visible(pos, window, sinks):
    """How many keys the query at `pos` sees."""
    if not window or pos < window:
        return pos + 1
    return window + min(sinks, pos + 1 - window)


def _keys(p, n, window, sinks):
    """How many keys any of the n rows from position p on sees."""
    lo = max(0, p + 1 - window) if window else 0
    return p + n - lo + min(sinks, lo)


def work(case):
    op, hkv = case["op"], case["hkv"]
    if op == "select":
        n = _lengths(case)
        kept = sum(min(x, case["keep"]) for x in n)
        seen = sum(max(0, x - case["recent"] - case["pin"]) for x in n if x > case["keep"])
        return {"bytes": 4 * hkv * (seen + kept), "flops": 0}
    if op == "compact":
        # of the rows that stay, those behind the first evicted one move (here: all but the pinned ones)
        moved = sum(max(0, case["keep"] - case["pin"]) for x in _lengths(case) if x > case["keep"])
        return {"bytes": hkv * moved * (4 + 2 * (2 * D * 2 + 4)), "flops": 0}
    hq = case["hq"]
    past, new, shared, starts = _requests(case)
    rows = sum(new)
    row_bytes = rows * hq * (2 * D * 2 + 4)
    if op == "shared":
        once = sum(shared[s] for s in starts[:-1])
        mine = sum(p + n - s for p, n, s in zip(past, new, shared))
        pairs = sum(_visible(q, 0, 0) for p, n in zip(past, new) for q in range(p, p + n))
        return {"bytes": (once + mine) * 2 * hkv * D * 2 + row_bytes + (8 * hkv * mine if case["scored"] else 0),
                "flops": 4 * D * hq * pairs}
    w, s = case["window"], case["sinks"]
    pairs = sum(_visible(q, w, s) for p, n in zip(past, new) for q in range(p, p + n))
    keys = sum(_keys(p, n, w, s) for p, n in zip(past, new))
    # chunks weigh every pair anew once the rows' sums are known: 2 D more to a pair
    few = max(new) * (hq // hkv) <= 16
    return {"bytes": keys * hkv * (2 * D * 2 + 8) + row_bytes, "flops": (4 if few else 6) * D * hq * pairs}


# ---------------------------------------------------------------- inputs
def _heads(gen, shape, dtype, scale=1.0):
    """Normal states with a few loud channels, as attention layers have them."""
    x = torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).mul_(scale)
    loud = torch.randint(0, D, (4,), generator=gen, device=DEV)
    x[..., loud] *= 3.0
    return x.to(dtype)


def _i32(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32).to(DEV)


def _table(case, seed, lengths, shared, starts):
    """Pages for requests of these lengths; the whole pages of a group's shared tokens are the same ones."""
    page = case["page"]
    width = max(1, max(-(-n // page) for n in lengths))
    common = [shared[s] // page for s in starts[:-1]] if any(shared) else []
    wanted = sum(-(-n // page) - s // page for n, s in zip(lengths, shared)) + sum(common)
    n_pages = wanted + 3
    order = np.random.RandomState(seed % (1 << 31)).permutation(n_pages).astype(np.int32)
    table = np.full((len(lengths), width), -1, dtype=np.int32)
    at = 0
    for g, c in enumerate(common):
        table[starts[g]:starts[g + 1], :c] = order[at:at + c]
        at += c
    for r, (n, s) in enumerate(zip(lengths, shared)):
        c, e = s // page, -(-n // page)
        table[r, c:e] = order[at:at + e - c]
        at += e - c
    return table, n_pages, order[at:]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed * 7919 + 23)
    op, page, hkv = case["op"], case["page"], case["hkv"]
    st = {"case": case}
    if op in ("select", "compact"):
        lengths = _lengths(case)
        past, new, shared, starts = lengths, [0] * len(lengths), [0] * len(lengths), [0]
    else:
        past, new, shared, starts = _requests(case)
        lengths = [p + n for p, n in zip(past, new)]
    table, n_pages, rest = _table(case, seed, lengths, shared, starts)
    st.update(table=_i32(table), kv_len=_i32(lengths))
    # accumulated weights: mostly small, a few tokens that many rows have looked at
    st["scores"] = torch.rand((n_pages, hkv, page), generator=gen, device=DEV).log_().mul_(-1.0).pow_(3.0).mul_(0.05)
    if op == "select":
        st["keep"], st["pin"] = _i32([case["keep"]] * case["req"]), _i32([case["pin"]] * case["req"])
        if own:
            import paper_2405_14256_b200 as zc
            dummy = torch.empty((n_pages, page, hkv, D), dtype=torch.float16, device=DEV)
            st["pool"] = zc.PagedKV(dummy, dummy, hkv, max_req=0, max_rows=0)
            st["kept"] = torch.empty((case["req"], hkv, case["keep"]), dtype=torch.int32, device=DEV)
        return st
    dt = TYPES[case["dtype"]]
    shape = (n_pages, hkv, page, D) if case["heads_first"] else (n_pages, page, hkv, D)
    view = (lambda t: t.transpose(1, 2)) if case["heads_first"] else (lambda t: t)
    st["k"], st["v"] = view(_heads(gen, shape, dt, 0.8)), view(_heads(gen, shape, dt))
    if op == "compact":
        _choose(st, case, gen, lengths)
        free = np.full(n_pages, -1, dtype=np.int32)
        free[n_pages - len(rest):] = rest
        st["free"], st["state"] = _i32(free), _i32([n_pages - len(rest), n_pages, 0])
        if own:
            import paper_2405_14256_b200 as zc
            st["pool"] = zc.PagedKV(st["k"], st["v"], hkv, max_req=0, max_rows=0)
            st["state_out"] = torch.zeros(3, dtype=torch.int32, device=DEV)
        return st
    if any(s % page for s in shared):
        # the page that a group's shared tokens do not fill is every request's own copy
        src, dst, row = [], [], []
        for g in range(len(starts) - 1):
            s = shared[starts[g]]
            for r in range(starts[g] + 1, starts[g + 1]):
                for i in range(s % page):
                    src.append(table[starts[g], s // page])
                    dst.append(table[r, s // page])
                    row.append(i)
        if src:
            src, dst, row = (_i32(x).long() for x in (src, dst, row))
            for pool in (st["k"], st["v"]):
                pool[dst, row] = pool[src, row]
    row_start = np.concatenate([[0], np.cumsum(new)])
    st.update(q=_heads(gen, (int(row_start[-1]), case["hq"], D), dt), row_start=_i32(row_start), max_new=max(new))
    if op == "shared":
        st.update(group_start=_i32(starts), shared_len=_i32([shared[s] for s in starts[:-1]]),
                  shared_max=max(shared), group_max=max(b - a for a, b in zip(starts, starts[1:])),
                  own_max=max(n - s for n, s in zip(lengths, shared)))
    else:
        st["pin"] = _i32([case["pin"]] * case["req"])
    if own:
        import paper_2405_14256_b200 as zc
        few = case["op"] == "shared" or max(new) * (case["hq"] // hkv) <= 16
        weighed = op == "scored" or case["scored"]
        st["pool"] = zc.PagedKV(st["k"], st["v"], case["hq"], max_req=len(new), max_rows=st["q"].shape[0],
                                shared=op == "shared", scored_rows=max(new) if weighed and few else 0)
        st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty(st["q"].shape[:-1], dtype=torch.float32, device=DEV)
    return st


def _choose(st, case, gen, lengths):
    """Tokens to keep, as a selection gives them: the first ones, the last ones, and others of every KV head's own."""
    req, hkv, keep = case["req"], case["hkv"], case["keep"]
    n = st["kv_len"].long()[:, None, None]
    at = torch.arange(max(lengths), device=DEV)
    rank = torch.rand((req, hkv, at.numel()), generator=gen, device=DEV)
    rank.masked_fill_((at < case["pin"]) | (at >= n - case["recent"]), 2.0).masked_fill_(at >= n, -1.0)
    top = rank.topk(min(keep, at.numel()), dim=-1).indices
    top = top.masked_fill(top >= n, at.numel()).sort(-1).values
    kept = torch.full((req, hkv, keep), -1, dtype=torch.int64, device=DEV)
    kept[..., :top.shape[-1]] = top
    length = torch.minimum(st["kv_len"], torch.tensor(keep, device=DEV))
    kept.masked_fill_(torch.arange(keep, device=DEV) >= length[:, None, None], -1)
    st["kept"], st["kept_len"] = kept.to(torch.int32), length.to(torch.int32)


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    op = case["op"]
    if op == "select":
        if own:
            kept, length = st["pool"].select(st["table"], st["kv_len"], st["scores"], st["keep"], case["recent"],
                                             first=st["pin"], kept=st["kept"])
        else:
            kept, length = _select(st, case)
        return {"kept": kept, "kept_len": length}
    if op == "compact":
        if own:
            state = st["pool"].compact(st["table"], st["kv_len"], st["kept"], st["kept_len"], scores=st["scores"],
                                       free_pages=st["free"], free_state=st["state"], free_out=st["state_out"])
        else:
            state = _compact(st, case)
        return {"k": st["k"], "v": st["v"], "scores": st["scores"], "free": st["free"], "state": state}
    if op == "shared":
        if own:
            out, lse = st["pool"].attention_shared(st["q"], st["table"], st["row_start"], st["kv_len"], st["max_new"],
                                                   st["group_start"], st["shared_len"],
                                                   scores=st["scores"] if case["scored"] else None, out=st["out"],
                                                   row_lse=st["lse"])
        else:
            out, lse = _shared(st, case)
        return {"out": out, "lse": lse, "scores": st["scores"]} if case["scored"] else {"out": out, "lse": lse}
    if own:
        out, lse = st["pool"].attention_scored(st["q"], st["table"], st["row_start"], st["kv_len"], st["max_new"],
                                               st["scores"], first=st["pin"], window=case["window"], sinks=case["sinks"],
                                               out=st["out"], row_lse=st["lse"])
    else:
        out, lse = _scored(st, case)
    return {"out": out, "lse": lse, "scores": st["scores"]}


def _dense(pages, table):
    """[requests, heads, tokens, D] of a pool in 32 bits, in table order."""
    x = pages[table.clamp(min=0).long()]
    return x.reshape(table.shape[0], -1, pages.shape[2], D).transpose(1, 2).float()


def _logits(q, k, seen):
    """Scaled logits (base 2) of q [b, hq, n, D] on k [b, hkv, s, D], -inf where not seen [b, n, s]."""
    b, hq, n, _ = q.shape
    x = torch.matmul(q.reshape(b, k.shape[1], -1, D), k.transpose(2, 3)).mul_(SCALE).reshape(b, hq, n, -1)
    return x.masked_fill_(~seen[:, None], -math.inf)


def _weighted(w, v):
    b, hq, n, s = w.shape
    return torch.matmul(w.reshape(b, v.shape[1], -1, s), v).reshape(b, hq, n, D)


def _chunks(st):
    """The requests' query rows, padded to the longest chunk, and where a row of the call is among them."""
    row_start, rows = st["row_start"].long(), st["q"].shape[0]
    i = torch.arange(st["max_new"], device=DEV)[None]
    q = st["q"][(row_start[:-1, None] + i).clamp(max=rows - 1)].transpose(1, 2).float()
    row = torch.arange(rows, device=DEV)
    req = torch.searchsorted(row_start[1:], row, right=True)
    return q, i, row_start[1:] - row_start[:-1], req, row - row_start[req]


def _add_weights(st, case, weights, first, since, begin):
    """Adds weights [requests, heads, rows, tokens] (tokens from position begin[r] on), summed over the rows and the query heads of
    a key head, to the tokens' scores; those from position since[r] on start from zero, those before first[r] are left."""
    b, hq, n, s = weights.shape
    total = weights.reshape(b, case["hkv"], -1, s).sum(2)
    pos = begin[:, None] + torch.arange(s, device=DEV)
    ok = (pos >= first[:, None]) & (pos < st["kv_len"].long()[:, None])
    req, tok = ok.nonzero(as_tuple=True)
    at = pos[req, tok]
    page, row = st["table"].long()[req, at // case["page"]], at % case["page"]
    old = torch.where((at >= since[req])[:, None], torch.zeros((), device=DEV), st["scores"][page, :, row])
    st["scores"][page, :, row] = old + total[req, :, tok]


def _scored(st, case):
    table, kv_len = st["table"], st["kv_len"].long()
    k, v = _dense(st["k"], table), _dense(st["v"], table)
    q, i, new, req, at = _chunks(st)
    j, p = torch.arange(k.shape[2], device=DEV), (kv_len - new)[:, None, None] + i[..., None]
    seen = j <= p
    if case["window"]:
        seen &= (j > p - case["window"]) | (j < case["sinks"])
    x = _logits(q, k, seen & (i < new[:, None])[..., None])
    top = x.amax(-1, keepdim=True).clamp_(min=-3e38)
    w = x.sub_(top).exp2_()
    total = w.sum(-1, keepdim=True)
    w = w.div_(total.clamp(min=1e-30))
    out, lse = _weighted(w, v), (top + total.log2()).squeeze(-1)
    _add_weights(st, case, w, st["pin"].long(), kv_len - new, torch.zeros_like(kv_len))
    return out[req, :, at].to(st["q"].dtype), lse[req, :, at]


def _shared(st, case):
    """The groups' rows over their shared keys, the requests' rows over their own, and the two joined."""
    table, kv_len, page = st["table"], st["kv_len"].long(), case["page"]
    start, shared = st["group_start"].long(), st["shared_len"].long()
    q, i, new, req, at = _chunks(st)
    n = q.shape[2]
    # shared keys: the requests of a group beside each other
    member = torch.arange(st["group_max"], device=DEV)[None]
    who = (start[:-1, None] + member).clamp(max=q.shape[0] - 1)
    gq = q[who].transpose(1, 2).reshape(start.numel() - 1, case["hq"], -1, D)
    gt = table[start[:-1], :-(-st["shared_max"] // page)]
    gk, gv = _dense(st["k"], gt), _dense(st["v"], gt)
    seen = (torch.arange(gk.shape[2], device=DEV) < shared[:, None])[:, None].expand(-1, gq.shape[2], -1)
    x = _logits(gq, gk, seen)
    top = x.amax(-1, keepdim=True)
    w = x.sub_(top).exp2_()
    group = torch.searchsorted(start[1:], torch.arange(q.shape[0], device=DEV), right=True)
    place = torch.arange(q.shape[0], device=DEV) - start[group]

    def back(t):      # of the groups' rows, those of each request
        return t.reshape(t.shape[0], case["hq"], -1, n, t.shape[-1])[group, :, place]
    o1, m1, s1 = back(_weighted(w, gv)), back(top), back(w.sum(-1, keepdim=True))
    # own keys, from the shared length on
    j = torch.arange(st["own_max"], device=DEV)
    pos = shared[group][:, None] + j
    ids = table.gather(1, (pos // page).clamp(max=table.shape[1] - 1)).clamp(min=0).long()
    k, v = (t[ids, pos % page].transpose(1, 2).float() for t in (st["k"], st["v"]))
    x = _logits(q, k, pos[:, None] <= ((kv_len - new)[:, None] + i)[..., None])
    m = torch.maximum(m1, x.amax(-1, keepdim=True))
    w = x.sub_(m).exp2_()
    f = (m1 - m).exp2_()
    total = s1 * f + w.sum(-1, keepdim=True)
    out, lse = (o1 * f + _weighted(w, v)) / total, (m + total.log2()).squeeze(-1)
    if case["scored"]:
        w = (w / total).masked_fill_((i >= new[:, None])[:, None, :, None], 0.0)
        _add_weights(st, case, w, shared[group], kv_len - new, shared[group])
    return out[req, :, at].to(st["q"].dtype), lse[req, :, at]


def _select(st, case):
    table, n = st["table"], st["kv_len"].long()[:, None, None]
    x = st["scores"][table.clamp(min=0).long()].transpose(1, 2).reshape(table.shape[0], case["hkv"], -1)
    at = torch.arange(x.shape[-1], device=DEV)
    stay = (at < st["pin"][:, None, None]) | (at >= n - case["recent"])
    x = x.masked_fill(stay, math.inf).masked_fill_(at >= n, -math.inf)
    order = x.sort(dim=-1, descending=True, stable=True).indices
    length = torch.minimum(st["kv_len"], st["keep"])
    rank = torch.empty_like(order).scatter_(-1, order, at.expand_as(order))
    keep = rank < length[:, None, None]
    kept = torch.full((x.shape[0], case["hkv"], case["keep"] + 1), -1, dtype=torch.int64, device=DEV)
    place = torch.where(keep, keep.cumsum(-1) - 1, case["keep"])
    kept.scatter_(-1, place, at.expand_as(place))
    return kept[..., :-1].to(torch.int32), length


def _compact(st, case):
    table, page, kept = st["table"].long(), case["page"], st["kept"].long()
    n, length = st["kv_len"].long(), st["kept_len"].long()
    i = torch.arange(kept.shape[-1], device=DEV)
    req, head, to = ((i < length[:, None, None]) & (length < n)[:, None, None] & (kept != i)).nonzero(as_tuple=True)
    src = kept[req, head, to]
    a = (table[req, src // page], src % page)
    b = (table[req, to // page], to % page)
    for pool in (st["k"], st["v"]):
        pool[b[0], b[1], head] = pool[a[0], a[1], head]
    st["scores"][b[0], head, b[1]] = st["scores"][a[0], head, a[1]]
    # the pages behind the kept tokens, request by request, in front of the free ones
    idx = torch.arange(table.shape[1], device=DEV)
    have, stay = (n + page - 1) // page, (length + page - 1) // page
    gone = table[(idx >= stay[:, None]) & (idx < have[:, None])]
    state = st["state"].long()
    begin = state[0] - gone.numel()
    st["free"][begin + torch.arange(gone.numel(), device=DEV)] = gone.to(torch.int32)
    return torch.stack([begin, state[1], torch.zeros_like(begin)]).to(torch.int32)


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    op = case["op"]
    if op == "select":
        return None          # whole numbers: they have to be equal
    st = prepare(case, seed)
    f64, page, hkv = torch.float64, case["page"], case["hkv"]
    ids, length = st["table"].tolist(), st["kv_len"].tolist()
    if op == "compact":
        outs = {"k": st["k"].to(f64).clone(), "v": st["v"].to(f64).clone(), "scores": st["scores"].to(f64).clone(),
                "free": None, "state": None}
        for r, n in enumerate(length):
            m = int(st["kept_len"][r])
            if m >= n:
                continue
            mine = torch.tensor(ids[r][:-(-n // page)], device=DEV)
            for h in range(hkv):
                src = st["kept"][r, h, :m].long()
                for name in ("k", "v"):
                    rows = outs[name][mine, :, h]                    # [pages, page, D], a copy
                    flat = rows.reshape(-1, D)
                    flat[:m] = flat[src].clone()
                    outs[name][mine, :, h] = flat.reshape(rows.shape)
                flat = outs["scores"][mine, h].reshape(-1)
                flat[:m] = flat[src].clone()
                outs["scores"][mine, h] = flat.reshape(-1, page)
        return outs
    group = case["hq"] // hkv
    start = st["row_start"].tolist()
    weighed = op == "scored" or case["scored"]
    scores = st["scores"].to(f64).clone()
    first = st["pin"].tolist() if op == "scored" else _requests(case)[2]
    window, sinks = case.get("window", 0), case.get("sinks", 0)
    out = torch.empty(st["q"].shape, dtype=f64, device=DEV)
    lse = torch.empty(st["q"].shape[:2], dtype=f64, device=DEV)
    for r, n in enumerate(length):
        a, e = start[r], start[r + 1]
        mine = torch.tensor(ids[r][:-(-n // page)], device=DEV)
        keys, values = (t[mine].flatten(0, 1)[:n].to(f64).transpose(0, 1) for t in (st["k"], st["v"]))
        i = torch.arange(n - (e - a), n, device=DEV)[:, None]
        j = torch.arange(n, device=DEV)[None]
        hidden = j > i
        if window:
            hidden |= (i - j >= window) & (j >= sinks)
        for h in range(hkv):
            q = st["q"][a:e, h * group:(h + 1) * group].to(f64)                      # rows, query heads, D
            x = (q @ keys[h].T / math.sqrt(D)).masked_fill(hidden[:, None], -math.inf)
            z = torch.logsumexp(x, -1)
            w = torch.exp(x - z[..., None])
            out[a:e, h * group:(h + 1) * group] = w @ values[h]
            lse[a:e, h * group:(h + 1) * group] = z / math.log(2)
            if weighed:
                t = torch.arange(first[r], n, device=DEV)
                at = (mine[t // page], torch.full_like(t, h), t % page)
                scores[at] = torch.where(t >= n - (e - a), 0.0, scores[at]) + w.sum((0, 1))[first[r]:]
    return {"out": out, "lse": lse, "scores": scores} if weighed else {"out": out, "lse": lse}
