"""Plain references, in 64 bits and Python integers, of the operators on full-precision pages, and
random steps to compare them on."""
from __future__ import annotations

import math

import numpy as np
import torch

D = 128


def tables(page, past, fresh, free_pages, state, table, n_rows):
    """Block tables and slots by the rule, request by request.  Returns the outputs as lists;
    `table` (a list of lists) is extended in place."""
    width = len(table[0])
    nxt, end = max(0, state[0]), min(state[1], len(free_pages))
    pages = lambda n: -(-n // page)  # noqa: E731
    taken = wanted = 0
    slots, pos = [-1] * n_rows, [-1] * n_rows
    row_start, kv_len = [0], []
    for r, (p, n) in enumerate(zip(past, fresh)):
        p, n = max(0, p), max(0, n)
        wanted += pages(p + n) - pages(p)
        for idx in range(min(pages(p), width), min(pages(p + n), width)):
            at = nxt + taken
            table[r][idx] = free_pages[at] if at < end else -1
            taken += 1
        for i in range(n):
            row = row_start[-1] + i
            if row < n_rows:
                t = p + i
                pos[row] = t
                pg = table[r][t // page] if t // page < width else -1
                slots[row] = pg * page + t % page if pg >= 0 else -1
        kv_len.append(p + n)
        row_start.append(row_start[-1] + n)
    got = min(taken, max(0, end - nxt))
    return kv_len, row_start, slots, pos, [nxt + got, end, wanted - got]


def rows_of_request(k, v, ids, n):
    """The first n tokens of a request, [n, heads, D] each, from pages [pages, page, heads, D]."""
    page = k.shape[1]
    ids = torch.as_tensor(ids[: -(-n // page)], device=k.device).long().clamp(min=0)
    return k[ids].flatten(0, 1)[:n], v[ids].flatten(0, 1)[:n]


def attend(q, k, v, first, window, sinks):
    """One head in 64 bits.  q [n, D] at positions first, first + 1, ...; k, v [s, D].  Returns out,
    the base-2 log-sum-exp, and what the tolerances are made of: the weighted mean of |v|, the largest
    sum of |q_i k_i| of a visible key (scaled, base 2), and the number of visible keys."""
    q, k, v = q.double(), k.double(), v.double()
    scale = math.log2(math.e) / math.sqrt(D)
    n, s = q.shape[0], k.shape[0]
    i = torch.arange(first, first + n, device=q.device)[:, None]
    j = torch.arange(s, device=q.device)[None]
    seen = (j <= i) & (((i - j) < window) | (j < sinks) if window else torch.ones_like(j, dtype=torch.bool))
    hidden = ~seen
    logit = (q @ k.T * scale).masked_fill(hidden, -math.inf)
    empty = hidden.all(1)
    top = torch.where(empty, torch.zeros((), dtype=torch.float64, device=q.device), logit.amax(1)) if s else torch.zeros(
        n, dtype=torch.float64, device=q.device)
    w = torch.exp2(logit - top[:, None])
    total = w.sum(1)
    w = w / total.clamp(min=1e-300)[:, None]
    vz = torch.where(torch.isfinite(v), v, torch.zeros_like(v))      # (only ever multiplied by a weight of 0)
    out, mean_abs = w @ vz, w @ vz.abs()
    lse = top + torch.log2(total)
    size = (q.abs() @ k.abs().T * scale).masked_fill(hidden, 0.0)
    size = torch.nan_to_num(size, nan=0.0, posinf=0.0)
    largest = size.amax(1) if s else torch.zeros_like(top)
    return out, lse, mean_abs, largest, seen.sum(1), total


def tolerances(dtype, out, mean_abs, largest, seen, total, vmax):
    """Derived bounds of |kernel - exact|.  u is half a step of the type.  Log-sum-exp (fp32 throughout):
    a logit is a sum of 128 exact products in fp32 in some order, off by at most 136 * 2^-24 of the sum of
    its terms' magnitudes; plus 2^-20 for the exponentials and the logarithm, and 2^-22 of its size.
    Output: each weight is off by u (its rounding to the type), and by ln 2 times twice the logits' error;
    fp16 weights below 2^-14 have an absolute step of 2^-24 against a sum of at least `total`; the stored
    output is off by u of its size (2^-25 below fp16's normal range)."""
    u = torch.finfo(dtype).eps / 2
    logit = 136 * 2.0 ** -24 * largest
    t_lse = logit + 2.0 ** -20 + 2.0 ** -22 * largest
    t_out = (u + 2 * math.log(2) * logit + 2.0 ** -18)[:, None] * mean_abs + u * out.abs() + 2.0 ** -24
    if dtype == torch.float16:
        t_out = t_out + (seen * 2.0 ** -25 * vmax / total.clamp(min=1.0))[:, None]
    return t_out, t_lse


def make_pages(gen, n_pages, page, heads, dtype, heads_first, device):
    def one():
        shape = (n_pages, heads, page, D) if heads_first else (n_pages, page, heads, D)
        x = torch.randn(shape, generator=gen, device=device)
        x[..., torch.randint(0, D, (3,), generator=gen, device=device)] *= 3.0
        x = x.to(dtype)
        return x.transpose(1, 2) if heads_first else x
    return one(), one()


def make_table(rng, lengths, page, width=None, spare=2):
    """A random assignment of pages: (table [R, width] numpy, number of pages)."""
    need = [-(-n // page) for n in lengths]
    n_pages = sum(need) + spare
    order = rng.permutation(n_pages)
    width = max(1, max(need)) if width is None else width
    table = np.full((len(lengths), width), -1, dtype=np.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return table, n_pages
