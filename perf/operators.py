"""The operators of the paged key/value cache, as cases that can be timed and compared.

A serving program keeps the keys and values of its running requests at full precision in pages
(blocks of `page_size` tokens) until a prompt is complete and is compressed.  Per step it
builds block tables and slot maps from the requests' lengths, writes the new rows into their
slots, attends from the new tokens to the cached ones (single tokens or chunks of a prompt, causal,
optionally a sliding window with a few first tokens that stay visible), and reads a finished
prompt's rows back as the dense tensors that the compression takes.

With `own` false, `run` computes each operator in elementary torch operations; with `own` true it
calls the framework.  Head counts, lengths and types are those of the repository's workloads
(64 x 4096, 128 x 8192, 1024 x 4096 and 32 x 32768 units x tokens, head dimension 128).
"""
import math
import random

import numpy as np
import torch

own = False

D = 128
DEV = "cuda:0"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases
def listed():
    return [
        # the plan of one step of eight requests that each generate a token: the smallest call of a serving loop
        dict(name="tables step 8", op="tables", req=8, page=16, past_lo=256, past_hi=1024, new_lo=1, new_hi=1, pad=0, mix=1),
        # admission of a large mixed batch: prompts' chunks beside single tokens, a padded row buffer
        dict(name="tables mixed 1024", op="tables", req=1024, page=16, past_lo=1, past_hi=16384, new_lo=1,
             new_hi=1024, pad=777, mix=2),
        # one generated token per request of workload 3, written into its page (rows of a joint q/k/v projection)
        dict(name="write step 16", op="write", dtype="fp16", req=16, hkv=8, page=64, past_lo=4096, past_hi=8192,
             new_lo=1, new_hi=1, heads_first=False, mix=3),
        # the prompts of workload 2, written at once, ragged by a little; pages with the heads outside the tokens
        dict(name="write prompts 8x4096", op="write", dtype="bf16", req=8, hkv=8, page=64, past_lo=1, past_hi=64,
             new_lo=3840, new_hi=4096, heads_first=True, mix=4),
        # workload 2's finished prompts, from pages to the dense tensors that prefill compression takes
        dict(name="read prompts 8x4096", op="read", dtype="bf16", req=8, hkv=8, page=16, past_lo=4096, past_hi=4096,
             new_lo=0, new_hi=0, heads_first=False, mix=5),
        # few short requests, one token each: latency
        dict(name="decode 4x512", op="attend", dtype="bf16", req=4, hq=32, hkv=8, page=16, past_lo=200, past_hi=512,
             new_lo=1, new_hi=1, window=0, sinks=0, heads_first=False, mix=6),
        # workload 4's heads (one query head per key head): the most bytes per step
        dict(name="decode mha 32x4096", op="attend", dtype="fp16", req=32, hq=32, hkv=32, page=64, past_lo=2048,
             past_hi=4096, new_lo=1, new_hi=1, window=0, sinks=0, heads_first=False, mix=7),
        # a chunk of a long prompt over workload 5's context
        dict(name="chunk 2048 at 30000", op="attend", dtype="bf16", req=1, hq=32, hkv=8, page=64, past_lo=30000, past_hi=30000,
             new_lo=2048, new_hi=2048, window=0, sinks=0, heads_first=True, mix=8),
        # a step that mixes chunks of every length with single tokens, ragged contexts
        dict(name="chunks mixed 16", op="attend", dtype="fp16", req=16, hq=32, hkv=8, page=16, past_lo=1, past_hi=8192,
             new_lo=1, new_hi=1024, window=0, sinks=0, heads_first=False, mix=9),
        # workload 3 with its model family's window of 4096 and four first tokens kept: single tokens
        dict(name="window decode 16x8192", op="attend", dtype="fp16", req=16, hq=32, hkv=8, page=64, past_lo=4100, past_hi=8192,
             new_lo=1, new_hi=1, window=4096, sinks=4, heads_first=False, mix=10),
        # the same window over chunks of long prompts
        dict(name="window chunks 4x1024", op="attend", dtype="bf16", req=4, hq=32, hkv=8, page=128, past_lo=0, past_hi=28000,
             new_lo=700, new_hi=1024, window=4096, sinks=4, heads_first=False, mix=11),
        # a whole prompt of workload 3 in dense tensors, under the same window
        dict(name="window prompt 8192", op="prompt", dtype="fp16", req=1, hq=32, hkv=8, l=8192, window=4096, sinks=4),
    ]


def _log(rng, lo, hi):
    """A whole number of lo .. hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(1, lo) - 0.499), math.log(hi + 0.499)))))))


def draw(rng):
    while True:
        op = rng.choice(["tables", "write", "read", "attend", "attend", "attend", "prompt"])
        mix = rng.randrange(1 << 30)
        if op == "tables":
            lo, hi = sorted((_log(rng, 1, 16384), _log(rng, 1, 16384)))
            nlo, nhi = sorted((_log(rng, 1, 1024), _log(rng, 1, 1024)))
            case = dict(op=op, req=_log(rng, 1, 1024), page=rng.choice([16, 32, 64, 128, 256]), past_lo=lo, past_hi=hi,
                        new_lo=nlo, new_hi=nhi, pad=rng.choice([0, 0, 1, 100, 777]), mix=mix)
            if case["req"] * nhi > 600000:
                continue
            return case
        dtype = rng.choice(["fp16", "bf16"])
        page = rng.choice([16, 32, 64, 128, 256])
        heads_first = rng.random() < 0.5
        if op in ("write", "read"):
            req = _log(rng, 1, 64)
            lo, hi = sorted((_log(rng, 1, 8192), _log(rng, 1, 8192)))
            hkv = rng.choice([1, 2, 4, 8, 32])
            case = dict(op=op, dtype=dtype, req=req, hkv=hkv, page=page, past_lo=0, past_hi=100, new_lo=lo, new_hi=hi,
                        heads_first=heads_first, mix=mix)
            if op == "read":     # dense tensors of one length
                case.update(past_lo=hi, past_hi=hi, new_lo=0, new_hi=0)
            if req * hi * hkv > 8 * 4096 * 8:
                continue
            return case
        hkv = rng.choice([1, 2, 4, 8, 8, 32])
        group = rng.choice([1, 2, 3, 4, 4, 5, 8]) if hkv < 32 else 1
        window, sinks = rng.choice([(0, 0), (0, 0), (0, 0), (_log(rng, 16, 8192), rng.choice([0, 1, 4, 100]))])
        if op == "prompt":
            case = dict(op=op, dtype=dtype, req=rng.choice([1, 1, 2, 4]), hq=hkv * group, hkv=hkv, l=_log(rng, 16, 8192),
                        window=_log(rng, 16, 8192), sinks=rng.choice([0, 1, 4, 100]))
        else:
            single = rng.random() < 0.5
            lo, hi = sorted((_log(rng, 1, 32768), _log(rng, 1, 32768)))
            nlo, nhi = (1, 1) if single else sorted((_log(rng, 1, 2048), _log(rng, 1, 2048)))
            case = dict(op=op, dtype=dtype, req=_log(rng, 1, 64 if single else 16), hq=hkv * group, hkv=hkv, page=page,
                        past_lo=lo, past_hi=hi, new_lo=nlo, new_hi=nhi, window=window, sinks=sinks,
                        heads_first=heads_first, mix=mix)
        # no dearer than the largest listed cases, and no larger a table of logits in the plain form
        w = work(case)
        n, s = (case["l"], case["l"]) if op == "prompt" else (case["new_hi"], case["past_hi"] + case["new_hi"])
        if w["flops"] <= 1.0e12 and w["bytes"] <= 1.49e9 and case["req"] * case["hq"] * n * s <= 2.2e9 \
                and case["req"] * case["hkv"] * s <= 5e6:
            return case


def _lengths(case):
    """Tokens already cached and new tokens of each request: the case's own, whatever the seed."""
    r = random.Random(case["mix"])
    draw_one = lambda lo, hi: lo if lo == hi else _log(r, lo, hi) if hi > 16 * max(1, lo) else r.randint(lo, hi)  # noqa: E731
    past = [draw_one(case["past_lo"], case["past_hi"]) for _ in range(case["req"])]
    new = [draw_one(case["new_lo"], case["new_hi"]) for _ in range(case["req"])]
    return past, new


def _visible(pos, window, sinks):
    """How many keys the query at `pos` sees."""
    if not window or pos < window:
        return pos + 1
    return window + min(sinks, pos + 1 - window)


def work(case):
    op = case["op"]
    if op == "prompt":
        b, l, w, s = case["req"], case["l"], case["window"], case["sinks"]
        seen = sum(_visible(p, w, s) for p in range(l))
        return {"bytes": b * l * (2 * case["hq"] + 2 * case["hkv"]) * D * 2 + 4 * b * l * case["hq"],
                "flops": 4 * D * b * case["hq"] * seen}
    past, new = _lengths(case)
    if op == "tables":
        pages = sum(-(-(p + n) // case["page"]) - -(-p // case["page"]) for p, n in zip(past, new))
        rows = sum(new) + case["pad"]
        return {"bytes": 4 * (3 * case["req"] + 1 + 2 * pages + 2 * rows + 6), "flops": 0}
    if op == "write":
        return {"bytes": sum(new) * (4 * case["hkv"] * D * 2 + 4), "flops": 0}
    if op == "read":
        return {"bytes": sum(past) * 4 * case["hkv"] * D * 2, "flops": 0}
    rows, w, s = sum(new), case["window"], case["sinks"]
    keys = seen = 0
    for p, n in zip(past, new):
        seen += sum(_visible(q, w, s) for q in range(p, p + n))
        lo = max(0, p + 1 - w) if w else 0              # first key in the first row's window
        keys += p + n - lo + min(s, lo)
    return {"bytes": keys * 2 * case["hkv"] * D * 2 + rows * case["hq"] * (2 * D * 2 + 4),
            "flops": 4 * D * case["hq"] * seen}


# ---------------------------------------------------------------- inputs
def _heads(gen, shape, dtype, scale=1.0):
    """Normal states with a few loud channels, as attention layers have them."""
    x = torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).mul_(scale)
    loud = torch.randint(0, D, (4,), generator=gen, device=DEV)
    x[..., loud] *= 3.0
    return x.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed * 7919 + 17)
    host = random.Random(seed * 104729 + 5)
    op = case["op"]
    st = {"case": case}
    if op == "prompt":
        b, l, dt = case["req"], case["l"], TYPES[case["dtype"]]
        st["q"] = _heads(gen, (b, case["hq"], l, D), dt)
        st["k"] = _heads(gen, (b, case["hkv"], l, D), dt, 0.8)
        st["v"] = _heads(gen, (b, case["hkv"], l, D), dt)
        if own:
            _handles(st)
        return st
    past, new = _lengths(case)
    page, n_req = case["page"], case["req"]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    width = max(1, max(-(-(p + n) // page) for p, n in zip(past, new)))
    held = [-(-(p + (0 if op == "tables" else n)) // page) for p, n in zip(past, new)]
    wanted = sum(-(-(p + n) // page) for p, n in zip(past, new))
    n_pages = wanted + 3
    order = np.random.RandomState(seed % (1 << 31)).permutation(n_pages).astype(np.int32)
    table = np.full((n_req, width), -1, dtype=np.int32)
    first = 0
    for r in range(n_req):
        table[r, :held[r]] = order[first:first + held[r]]
        first += held[r]
    st["table"] = i32(table)
    if op == "tables":
        start = host.randrange(0, 3)
        st.update(past=i32(past), new=i32(new), free=i32(np.concatenate([np.zeros(start, np.int32), order[first:]])),
                  state=i32([start, start + n_pages - first, 0]), rows=sum(new) + case["pad"])
        if own:
            _handles(st)
        return st
    dt, hkv = TYPES[case["dtype"]], case["hkv"]
    shape = (n_pages, hkv, page, D) if case["heads_first"] else (n_pages, page, hkv, D)
    view = (lambda t: t.transpose(1, 2)) if case["heads_first"] else (lambda t: t)
    st["k"], st["v"] = view(_heads(gen, shape, dt, 0.8)), view(_heads(gen, shape, dt))
    hq = case.get("hq", hkv)
    if op == "read":
        st["l"] = past[0]
        if own:
            _handles(st)
        return st
    row_start = np.concatenate([[0], np.cumsum(new)])
    rows = int(row_start[-1])
    if op == "write":
        joint = _heads(gen, (rows, 2 * hkv, D), dt)      # keys and values side by side, as a joint projection leaves them
        st["k_rows"], st["v_rows"] = joint[:, :hkv], joint[:, hkv:]
        req = np.repeat(np.arange(n_req), new)
        pos = np.asarray(past)[req] + np.arange(rows) - row_start[req]
        st["slots"] = i32(table[req, pos // page].astype(np.int64) * page + pos % page)
    else:
        st.update(q=_heads(gen, (rows, hq, D), dt), row_start=i32(row_start), max_new=max(new),
                  kv_len=i32([p + n for p, n in zip(past, new)]))
    if own:
        _handles(st)
    return st


def _handles(st):
    """What a program makes once beside its data: the handle of its pages or of its cache, and the buffers
    that every step writes its results to."""
    import paper_2405_14256_b200 as zc
    case = st["case"]
    if case["op"] == "tables":
        st["step"] = zc.StepTables(case["req"], st["rows"], device=DEV)
    elif case["op"] == "prompt":
        st["cache"] = zc.ZipCache(st["q"].dtype, case["req"], case["hq"], case["hkv"], case["l"], 1, 0.4, device=DEV)
    else:
        st["pool"] = zc.PagedKV(st["k"], st["v"], case.get("hq", case["hkv"]), max_req=case["req"],
                                max_rows=st["q"].shape[0] if "q" in st else 0)
    if "q" in st:
        st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty(st["q"].shape[:-1], dtype=torch.float32, device=DEV)


# ---------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    op = case["op"]
    if op == "tables":
        if own:
            step = st["step"]
            step.build(case["page"], st["past"], st["new"], st["free"], st["state"], st["table"])
            kv_len, row_start, slots, pos, state = step.kv_len, step.row_start, step.slots, step.pos, step.free_state
        else:
            kv_len, row_start, slots, pos, state = _tables(st, case["page"])
        return {"table": st["table"], "kv_len": kv_len, "row_start": row_start, "slots": slots, "pos": pos, "state": state}
    if op == "write":
        if own:
            st["pool"].write(st["k_rows"], st["v_rows"], st["slots"])
        else:
            slots = st["slots"].long()
            at = (slots // case["page"], slots % case["page"])
            st["k"][at] = st["k_rows"]
            st["v"][at] = st["v_rows"]
        return {"k": st["k"], "v": st["v"]}
    if op == "read":
        if own:
            k, v = st["pool"].read(st["table"], st["l"])
        else:
            k, v = (_dense(t, st["table"])[:, :st["l"]].transpose(1, 2).contiguous() for t in (st["k"], st["v"]))
        return {"k": k, "v": v}
    if op == "prompt":
        if own:
            out, lse = st["cache"].prefill_attention_window(st["q"], st["k"], st["v"], case["window"], case["sinks"],
                                                               out=st["out"], row_lse=st["lse"])
        else:
            l = case["l"]
            pos = torch.arange(l, device=DEV)[None].expand(case["req"], l)
            out, lse = _attend(st["q"].float(), st["k"].float(), st["v"].float(), pos, case["window"], case["sinks"])
            out = out.to(st["q"].dtype)
        return {"out": out, "lse": lse}
    if own:
        out, lse = st["pool"].attention(st["q"], st["table"], st["row_start"], st["kv_len"], st["max_new"],
                                        window=case["window"], sinks=case["sinks"], out=st["out"], row_lse=st["lse"])
    else:
        out, lse = _paged(st, case)
    return {"out": out, "lse": lse}


def _tables(st, page):
    """Pages of the free list to the requests in their order, then every new row's position and slot."""
    table, i64 = st["table"], torch.int64
    past, new, state = st["past"].to(i64), st["new"].to(i64), st["state"].to(i64)
    had, total = (past + page - 1) // page, past + new
    need = (total + page - 1) // page - had
    last = torch.cumsum(need, 0)
    at = torch.arange(table.shape[1], device=DEV)[None] - had[:, None]
    index = state[0] + (last - need)[:, None] + at
    granted = torch.where(index < state[1], st["free"][index.clamp(0, st["free"].numel() - 1)], -1)
    table.copy_(torch.where((at >= 0) & (at < need[:, None]), granted, table))
    end = torch.cumsum(new, 0)
    row = torch.arange(st["rows"], device=DEV)
    req = torch.searchsorted(end, row, right=True).clamp(max=past.numel() - 1)
    pos = torch.where(row < end[-1], past[req] + row - (end - new)[req], -1)
    held = table[req, pos.clamp(min=0) // page].to(i64)
    slots = torch.where((pos >= 0) & (held >= 0), held * page + pos % page, -1)
    took = torch.minimum(last[-1], state[1] - state[0])
    row_start = torch.cat([torch.zeros(1, dtype=i64, device=DEV), end])
    out = torch.stack([state[0] + took, state[1], last[-1] - took])
    return tuple(x.to(torch.int32) for x in (total, row_start, slots, pos, out))


def _dense(pages, table):
    """[requests, tokens, heads, D] of a pool, in table order."""
    x = pages[table.clamp(min=0).long()]
    return x.reshape(table.shape[0], -1, pages.shape[2], D)


def _attend(q, k, v, pos, window, sinks):
    """softmax(q k^T / sqrt(D)) v over the keys that each query sees, and the base-2 log-sum-exp.
    q [b, hq, n, D], k and v [b, hkv, s, D] in 32 bits, pos [b, n] the queries' positions."""
    b, hq, n, _ = q.shape
    hkv, s = k.shape[1:3]
    logits = torch.matmul(q.reshape(b, hkv, -1, D), k.transpose(2, 3)).mul_(math.log2(math.e) / math.sqrt(D))
    logits = logits.reshape(b, hq, n, s)
    j, p = torch.arange(s, device=DEV), pos[..., None]
    seen = j <= p
    if window:
        seen &= (j > p - window) | (j < sinks)
    logits.masked_fill_(~seen[:, None], -math.inf)
    top = logits.amax(-1, keepdim=True).clamp_(min=-3e38)
    weights = logits.sub_(top).exp2_()
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights.reshape(b, hkv, -1, s), v).reshape(b, hq, n, D).div_(total)
    return out, (top + total.log2()).squeeze(-1)


def _paged(st, case):
    table, row_start, kv_len = st["table"], st["row_start"].long(), st["kv_len"].long()
    rows, n = st["q"].shape[0], st["max_new"]
    k, v = (_dense(t, table).transpose(1, 2).float() for t in (st["k"], st["v"]))
    i = torch.arange(n, device=DEV)[None]
    new = (row_start[1:] - row_start[:-1])[:, None]
    q = st["q"][(row_start[:-1, None] + i).clamp(max=rows - 1)].transpose(1, 2).float()      # padded to the longest chunk
    out, lse = _attend(q, k, v, kv_len[:, None] - new + i, case["window"], case["sinks"])
    row = torch.arange(rows, device=DEV)
    req = torch.searchsorted(row_start[1:], row, right=True)
    at = row - row_start[req]
    return out[req, :, at].to(st["q"].dtype), lse[req, :, at]


# ---------------------------------------------------------------- 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "tables":
        return None          # whole numbers: they have to be equal
    f64 = torch.float64
    if op == "write":
        k, v = st["k"].to(f64).clone(), st["v"].to(f64).clone()
        for pool, rows in ((k, st["k_rows"]), (v, st["v_rows"])):
            for r, slot in zip(rows.to(f64).cpu().unbind(0) if rows.shape[0] < 64 else [], st["slots"].tolist()):
                pool[slot // case["page"], slot % case["page"]] = r.to(DEV)
            if rows.shape[0] >= 64:
                flat = pool.transpose(1, 2).reshape(-1, D).clone() if case["heads_first"] else pool.reshape(-1, D).clone()
                s, h = st["slots"].long()[:, None], torch.arange(case["hkv"], device=DEV)[None]
                p = case["page"]
                at = (s // p * case["hkv"] + h) * p + s % p if case["heads_first"] else s * case["hkv"] + h
                flat.index_copy_(0, at.reshape(-1), rows.to(f64).reshape(-1, D))
                pool.copy_(flat.reshape(pool.shape[0], case["hkv"], p, D).transpose(1, 2) if case["heads_first"]
                           else flat.reshape(pool.shape))
        return {"k": k, "v": v}
    if op == "read":
        outs = []
        for pool in (st["k"], st["v"]):
            per = [torch.cat([pool[i] for i in ids if i >= 0], 0)[:st["l"]].to(f64) for ids in st["table"].tolist()]
            outs.append(torch.stack(per).permute(0, 2, 1, 3))
        return {"k": outs[0], "v": outs[1]}
    group = case["hq"] // case["hkv"]
    if op == "prompt":
        out = torch.empty(st["q"].shape, dtype=f64, device=DEV)
        lse = torch.empty(st["q"].shape[:3], dtype=f64, device=DEV)
        for b in range(case["req"]):
            for h in range(case["hq"]):
                out[b, h], lse[b, h] = _one_head(st["q"][b, h], st["k"][b, h // group], st["v"][b, h // group], 0, case)
        return {"out": out, "lse": lse}
    start, length, ids = st["row_start"].tolist(), st["kv_len"].tolist(), st["table"].tolist()
    out = torch.empty(st["q"].shape, dtype=f64, device=DEV)
    lse = torch.empty(st["q"].shape[:2], dtype=f64, device=DEV)
    for r in range(case["req"]):
        a, e, n = start[r], start[r + 1], length[r]
        own_pages = torch.tensor(ids[r][:-(-n // case["page"])], device=DEV)
        keys, values = (t[own_pages].flatten(0, 1)[:n] for t in (st["k"], st["v"]))
        for h in range(case["hq"]):
            out[a:e, h], lse[a:e, h] = _one_head(st["q"][a:e, h], keys[:, h // group], values[:, h // group], n - (e - a), case)
    return {"out": out, "lse": lse}


def _one_head(q, k, v, first, case):
    """One head's attention in 64 bits; the query rows sit at positions first, first + 1, ..."""
    score = q.double() @ k.double().T / math.sqrt(D)
    i = torch.arange(first, first + q.shape[0], device=DEV)[:, None]
    j = torch.arange(k.shape[0], device=DEV)[None]
    hidden = j > i
    if case["window"]:
        hidden |= (i - j >= case["window"]) & (j >= case["sinks"])
    score[hidden.expand_as(score)] = -math.inf
    lse = torch.logsumexp(score, -1)
    return torch.exp(score - lse[:, None]) @ v.double(), lse / math.log(2)
