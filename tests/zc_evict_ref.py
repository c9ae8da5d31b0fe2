"""Plain references, in 64 bits and Python integers, of the weights that attention gives cached tokens, of the selection
by them and of the compaction of pages; and random requests that begin alike."""
from __future__ import annotations

import math

import numpy as np
import torch

import zc_paged_ref as ref

D = 128


def weights(q, k, first, window, sinks):
    """One query head in 64 bits: q [n, D] at positions first, ...; k [s, D].  Returns the weights [n, s] and a bound of
    the relative error of each row's: with the logits' and the log-sum-exp's own (zc_paged_ref.tolerances), 2^-20 for the
    exponential."""
    v = torch.zeros_like(k)
    _, lse, mean_abs, largest, seen, total = ref.attend(q, k, v, first, window, sinks)
    _, t_lse = ref.tolerances(torch.float16, mean_abs[:, None], mean_abs[:, None], largest, seen, total, 1.0)
    scale = math.log2(math.e) / math.sqrt(D)
    n, s = q.shape[0], k.shape[0]
    i = torch.arange(first, first + n, device=q.device)[:, None]
    j = torch.arange(s, device=q.device)[None]
    shown = (j <= i) & (((i - j) < window) | (j < sinks) if window else torch.ones_like(j, dtype=torch.bool))
    x = torch.nan_to_num(q.double() @ k.double().T * scale)
    w = torch.where(shown, torch.exp2(x - lse[:, None]), torch.zeros((), dtype=torch.float64, device=q.device))
    rel = math.log(2) * (136 * 2.0 ** -24 * largest + t_lse) + 2.0 ** -20
    return w, rel


def add_weights(scores, q, kp, table, row_start, kv_len, first, window, sinks):
    """What scores [pages, heads, page] (float32) become, in 64 bits, and how far off fp32 sums may be."""
    page, hkv = kp.shape[1], kp.shape[2]
    G = q.shape[1] // hkv
    want = scores.double().clone()
    tol = torch.zeros_like(want)
    for r, n in enumerate(kv_len):
        a, e = row_start[r], row_start[r + 1]
        if e <= a or n <= 0:
            continue
        k, _ = ref.rows_of_request(kp, kp, table[r], n)
        p0 = n - (e - a)
        j = torch.arange(n, device=q.device)
        ids = torch.as_tensor(table[r], device=q.device).long()[j // page]
        i = torch.arange(p0, n, device=q.device)[:, None]
        seen = (j <= i) & (((i - j) < window) | (j < sinks) if window else torch.ones_like(j, dtype=torch.bool))
        use = seen.any(0) & (j >= first[r])
        for h in range(hkv):
            total, off = torch.zeros(n, dtype=torch.float64, device=q.device), torch.zeros(n, dtype=torch.float64, device=q.device)
            for g in range(G):
                w, rel = weights(q[a:e, h * G + g], k[:, h], p0, window, sinks)
                total += w.sum(0)
                off += (w * rel[:, None]).sum(0)
            # sums of (e - a) G weights, one after the other, and of the old score
            off += total * ((e - a) * G + 2) * 2.0 ** -24 + 2.0 ** -100
            at = (ids[use], torch.full_like(ids[use], h), (j % page)[use])
            old = torch.where(j >= p0, torch.zeros((), dtype=torch.float64, device=q.device), scores.double()[ids, h, j % page])[use]
            want[at] = old + total[use]
            tol[at] = off[use] + (old + total[use]).abs() * 2.0 ** -23
    return want, tol


def select(scores, table, page, kv_len, keep, recent, first, max_keep):
    """Position lists by the rule, in Python: kept[r][h] and the new lengths."""
    n_pages, hkv, _ = scores.shape
    host = scores.cpu().numpy()
    kept, lens = [], []
    for r, n in enumerate(kv_len):
        n = min(max(n, 0), len(table[r]) * page)
        f = min(max(first[r], 0), n)
        rc = min(recent, n - f)
        budget = max(min(max(keep[r], 0), max_keep), f + rc)
        whole = budget >= n or budget > max_keep
        m = n if whole else budget
        lens.append(m)
        lists = []
        for h in range(hkv):
            if whole:
                pos = list(range(min(n, max_keep)))
            else:
                def key(t):
                    p = table[r][t // page]
                    x = float(host[p, h, t % page]) if 0 <= p < n_pages else math.nan
                    return (x == x, 0.0 if x != x else x)
                cand = sorted(range(f, n - rc), key=key, reverse=True)      # (stable: ties stay in order)
                pos = sorted(list(range(f)) + cand[: m - f - rc] + list(range(n - rc, n)))
            lists.append(pos + [-1] * (max_keep - len(pos)))
        kept.append(lists)
    return kept, lens


def compact(k, v, scores, table, page, kv_len, kept, lens, max_keep):
    """Copies of the pools with the kept rows in front."""
    k2, v2, s2 = k.clone(), v.clone(), scores.clone()
    for r, (n, m) in enumerate(zip(kv_len, lens)):
        if m >= n or m > max_keep:
            continue
        for h in range(k.shape[2]):
            src = np.asarray(kept[r][h][:m], dtype=np.int64)
            dst = np.arange(m)
            t = np.asarray(table[r])
            a, b = (torch.as_tensor(t[x // page].astype(np.int64), device=k.device) for x in (src, dst))
            i, j = (torch.as_tensor((x % page).astype(np.int64), device=k.device) for x in (src, dst))
            k2[b, j, h], v2[b, j, h], s2[b, h, j] = k[a, i, h], v[a, i, h], scores[a, h, i]
    return k2, v2, s2


def freed(table, page, kv_len, lens, free_pages, state, max_keep):
    """The free list after the pages behind the kept tokens are put back, and its state."""
    gone = []
    for r, (n, m) in enumerate(zip(kv_len, lens)):
        if m < n and m <= max_keep:
            gone += [int(x) for x in table[r][-(-m // page): -(-n // page)]]
    free = list(free_pages)
    nxt = min(max(state[0], 0), len(free))
    for i, p in enumerate(gone):
        at = nxt - len(gone) + i
        if at >= 0:
            free[at] = p
    return free, [max(0, nxt - len(gone)), min(state[1], len(free)), max(0, len(gone) - nxt)]


def make_groups(rng, page, groups, shared, own, alone=0):
    """Tables of requests that begin alike: groups[g] requests share shared[g] tokens, then have lengths own (one after the
    other); `alone` requests behind them share nothing.  Returns table, lengths, group starts, pages, and pairs of (page
    to copy from, to, rows) for the pages that the shared tokens do not fill."""
    lens, sh, starts = [], [], [0]
    own = list(own)
    for n, s in zip(groups, shared):
        lens += [s + own.pop(0) for _ in range(n)]
        sh += [s] * n
        starts.append(len(lens))
    lens += [own.pop(0) for _ in range(alone)]
    sh += [0] * alone
    width = max(1, max(-(-n // page) for n in lens))
    need = sum(-(-n // page) - s // page for n, s in zip(lens, sh)) + sum(s // page for s in shared)
    order = rng.permutation(need + 2)
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for g, s in enumerate(shared):
        table[starts[g]:starts[g + 1], : s // page] = order[at:at + s // page]
        at += s // page
    copies = []
    for r, (n, s) in enumerate(zip(lens, sh)):
        c, e = s // page, -(-n // page)
        table[r, c:e] = order[at:at + e - c]
        at += e - c
    for g, s in enumerate(shared):
        if s % page:
            copies += [(int(table[starts[g], s // page]), int(table[r, s // page]), s % page)
                       for r in range(starts[g] + 1, starts[g + 1])]
    return table, lens, starts, need + 2, copies
