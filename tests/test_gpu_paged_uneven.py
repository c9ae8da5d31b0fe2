"""Pages that are shared and thinned out, on the GPU, where a server's state is uneven: idle requests in a group, queries
and keys that are not numbers, tables with entries that are no page, budgets beyond the list, slots that two requests score,
calls without requests."""
import math

import numpy as np
import pytest
import torch

import zc_evict_ref as er
import zc_paged_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def zc():
    import paper_2405_14256_b200 as mod
    mod.load_library()
    return mod


def i32(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32).to(DEV)


def settled(zc):
    torch.cuda.synchronize()
    assert zc.zc_device_status() == 0


# ---------------------------------------------------------------- idle requests
def wide(table, page, hkv, n_groups):
    """The table with so many empty columns that sharing may pay by its width."""
    spare = len(table) - min(n_groups, len(table))
    width = int(1e8 / max(1, spare * hkv * 512 * page)) + 1
    return np.pad(table, ((0, 0), (0, max(0, width - table.shape[1]))), constant_values=-1)


IDLE = [
    # the first request of each group has ended; in the second case two of them, and a group is idle as a whole
    dict(hq=32, hkv=32, page=16, groups=[5, 4], shared=[1200, 900], new=[0, 1, 2, 1, 1, 0, 2, 1, 1]),
    dict(hq=32, hkv=8, page=64, groups=[12, 3, 9], shared=[2000, 700, 1500],
         new=[0, 0] + [1] * 10 + [0] * 3 + [0] + [1, 0] * 4),
    # more requests than are planned in shared memory
    dict(hq=2, hkv=1, page=16, groups=[800, 60], shared=[640, 700], new=[0] * 40 + [1] * 760 + [0] + [1] * 59),
]


@pytest.mark.parametrize("left", ["cleared", "reused"])
@pytest.mark.parametrize("scored", [False, True])
@pytest.mark.parametrize("kw", IDLE)
def test_a_group_goes_on_when_its_first_requests_have_ended(zc, kw, scored, left):
    """Their table rows may be anything by then: empty, or another conversation's pages."""
    hq, hkv, page, new = kw["hq"], kw["hkv"], kw["page"], kw["new"]
    rng, gen, dt = np.random.RandomState(3), torch.Generator(device=DEV).manual_seed(4), torch.bfloat16
    n_req = len(new)
    table, kv, starts, n_pages, copies = er.make_groups(rng, page, kw["groups"], kw["shared"], [5 + 7 * i % 90 for i in range(n_req)])
    table = wide(table, page, hkv, len(kw["groups"]))
    k, v = ref.make_pages(gen, n_pages + 9, page, hkv, dt, False, DEV)
    for src, dst, rows in copies:
        for pool in (k, v):
            pool[dst, :rows] = pool[src, :rows]
    for r in range(n_req):
        if new[r] == 0:
            table[r] = -1
            kv[r] = 0
            if left == "reused":
                table[r, :9] = np.arange(n_pages, n_pages + 9)
                kv[r] = 8 * page
    row_start = [0] + np.cumsum(new).tolist()
    rows, most = row_start[-1], max(new)
    q = torch.randn(rows, hq, D, generator=gen, device=DEV).to(dt)
    pool = zc.PagedKV(k, v, hq, max_req=n_req, max_rows=rows, shared=True, scored_rows=most)
    scores = torch.rand((n_pages + 9, hkv, page), generator=gen, device=DEV)
    before = scores.clone()
    out, lse = pool.attention_shared(q, i32(table), i32(row_start), i32(kv), most, i32(starts), i32(kw["shared"]),
                                     scores=scores if scored else None)
    settled(zc)
    vmax = v.abs().max().double()
    for r in range(0, n_req, 1 if n_req < 100 else 37):
        a, e = row_start[r], row_start[r + 1]
        if a == e:
            continue
        kr, vr = ref.rows_of_request(k, v, table[r], kv[r])
        for h in range(hq):
            g = h // (hq // hkv)
            o, l, mean_abs, largest, seen, total = ref.attend(q[a:e, h], kr[:, g], vr[:, g], kv[r] - (e - a), 0, 0)
            t_out, t_lse = ref.tolerances(dt, o, mean_abs, largest, seen, total, vmax)
            assert ((out[a:e, h].double() - o).abs() <= t_out).all() and ((lse[a:e, h].double() - l).abs() <= t_lse).all(), (r, h)
    if scored and n_req < 100:
        first = [s for s, n in zip(kw["shared"], kw["groups"]) for _ in range(n)]
        want, tol = er.add_weights(before, q, k, table, row_start, kv, first, 0, 0)
        assert ((scores.double() - want).abs() <= tol).all()


# ---------------------------------------------------------------- what is not a number
def poisoned(q, kp, table, row_start, kv_len, window, sinks):
    """[pages, heads, page] bool: slots that a row sees one of whose logits is NaN or +inf in 64 bits, where its weights are NaN."""
    n_pages, page, hkv, _ = kp.shape
    G = q.shape[1] // hkv
    bad = torch.zeros((n_pages, hkv, page), dtype=torch.bool, device=DEV)
    for r, n in enumerate(kv_len):
        a, e = row_start[r], row_start[r + 1]
        if e <= a or n <= 0:
            continue
        k, _ = ref.rows_of_request(kp, kp, table[r], n)
        j, p0 = torch.arange(n, device=DEV), n - (e - a)
        i = torch.arange(p0, n, device=DEV)[:, None]
        seen = (j <= i) & (((i - j) < window) | (j < sinks) if window else torch.ones_like(j, dtype=torch.bool))
        ids = torch.as_tensor(table[r], device=DEV).long()[j // page]
        for h in range(hkv):
            for g in range(G):
                x = q[a:e, h * G + g].double() @ k[:, h].double().T
                row = (seen & (x.isnan() | (x == math.inf))).any(1)
                at = (seen & row[:, None]).any(0)
                bad[ids[at], h, (j % page)[at]] = True
    return bad


NAN = [
    # single tokens, few rows, chunks; under a window rows that do not see the key keep their weights
    dict(hq=8, hkv=2, page=16, past=[100, 300, 33], new=[1, 1, 1]),
    dict(hq=4, hkv=2, page=16, past=[100, 300, 33], new=[3, 1, 4]),
    dict(hq=18, hkv=2, page=16, past=[100, 40], new=[1, 1]),
    dict(hq=8, hkv=2, page=64, past=[100, 300, 3000], new=[1, 1, 1], window=200, sinks=4),
    dict(hq=8, hkv=2, page=16, past=[100, 300, 0], new=[40, 130, 300]),
    dict(hq=6, hkv=2, page=64, past=[500, 20], new=[200, 150], window=90, sinks=3),
]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("where,value", [("key", math.nan), ("query", math.nan), ("query", math.inf), ("key", math.inf)])
@pytest.mark.parametrize("kw", NAN)
def test_weights_of_rows_that_are_not_numbers_are_none(zc, kw, where, value, dtype):
    """A row with a logit that is no finite number has no softmax: its weights are NaN for every token that it sees, and
    no other token's score is touched by it."""
    hq, hkv, page, past, new = (kw[x] for x in ("hq", "hkv", "page", "past", "new"))
    window, sinks = kw.get("window", 0), kw.get("sinks", 0)
    rng, gen, dt = np.random.RandomState(1), torch.Generator(device=DEV).manual_seed(2), TYPES[dtype]
    kv = [p + n for p, n in zip(past, new)]
    table, n_pages = ref.make_table(rng, kv, page)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
    row_start = [0] + np.cumsum(new).tolist()
    q = torch.randn(row_start[-1], hq, D, generator=gen, device=DEV).to(dt)
    k2, q2 = k.clone(), q.clone()
    if where == "key":
        q[..., 7] = q[..., 7].abs() + 0.5                         # (+inf then makes +inf of every logit)
        q2 = q.clone()
        for r, t in ((0, past[0] // 2), (1, kv[1] - 1)):      # in the past, and the newest token's own
            k2[int(table[r][t // page]), t % page, r % hkv, 7] = value
    else:
        q2[0, 0, 5] = value
        q2[row_start[1] + new[1] // 2, hq - 1, 100] = value
    start = torch.rand((n_pages, hkv, page), generator=gen, device=DEV)
    most = max(new)
    few = most * (hq // hkv) <= 16
    scores = []
    for keys, queries in ((k, q), (k2, q2)):
        pool = zc.PagedKV(keys, v, hq, max_req=len(kv), max_rows=row_start[-1], scored_rows=most if few else 0)
        s = start.clone()
        pool.attention_scored(queries, i32(table), i32(row_start), i32(kv), most, s, window=window, sinks=sinks)
        settled(zc)
        scores.append(s)
    clean, got = scores
    bad = poisoned(q2, k2, table, row_start, kv, window, sinks)
    assert bad.any() and not bad.all()
    assert torch.isnan(got[bad]).all()
    # the same rows weigh the others: each weight off by 2^-18 of it at most in either call, sums by their roundings
    tol = clean * (2 * 2.0 ** -18 + 2 * (most * (hq // hkv) + 2) * 2.0 ** -24)
    assert ((got - clean).abs() <= tol)[~bad].all()


@pytest.mark.parametrize("past,new", [([100, 30], [1, 2]), ([100, 30], [40, 130])])
def test_a_logit_of_minus_infinity_is_a_weight_of_zero(zc, past, new):
    hq, hkv, page = 8, 2, 16
    gen, dt = torch.Generator(device=DEV).manual_seed(2), torch.bfloat16
    kv = [p + n for p, n in zip(past, new)]
    table, n_pages = ref.make_table(np.random.RandomState(1), kv, page)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
    row_start = [0] + np.cumsum(new).tolist()
    q = torch.randn(row_start[-1], hq, D, generator=gen, device=DEV).to(dt)
    q[..., 7] = q[..., 7].abs() + 0.5
    at = (int(table[1][1]), 3, 1)                                 # token 19 of request 1, KV head 1
    k[at][7] = -math.inf
    start = torch.rand((n_pages, hkv, page), generator=gen, device=DEV)
    scores = start.clone()
    pool = zc.PagedKV(k, v, hq, max_req=2, max_rows=row_start[-1], scored_rows=2)
    pool.attention_scored(q, i32(table), i32(row_start), i32(kv), max(new), scores)
    settled(zc)
    want, tol = er.add_weights(start, q, k, table, row_start, kv, [0, 0], 0, 0)
    assert ((scores.double() - want).abs() <= tol).all()
    assert scores[at[0], at[2], at[1]] == (start[at[0], at[2], at[1]] if past[1] > 19 else 0)


def test_shared_weights_of_rows_that_are_not_numbers(zc):
    rng, gen, dt = np.random.RandomState(1), torch.Generator(device=DEV).manual_seed(2), torch.bfloat16
    hq, hkv, page = 8, 2, 16
    table, kv, starts, n_pages, copies = er.make_groups(rng, page, [6], [960], [30, 1, 70, 5, 16, 17])
    table = wide(table, page, hkv, 1)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
    q = torch.randn(6, hq, D, generator=gen, device=DEV).to(dt)
    q2 = q.clone()
    q2[2, 5, 3] = math.nan
    pool = zc.PagedKV(k, v, hq, max_req=6, max_rows=6, shared=True, scored_rows=1)
    got = []
    for x in (q, q2):
        s = torch.zeros((n_pages, hkv, page), device=DEV)
        pool.attention_shared(x, i32(table), i32(range(7)), i32(kv), 1, i32(starts), i32([960]), scores=s)
        settled(zc)
        got.append(s)
    bad = torch.zeros_like(got[0], dtype=torch.bool)
    for t in range(960, kv[2]):
        bad[int(table[2][t // page]), 1, t % page] = True
    assert torch.isnan(got[1][bad]).all() and torch.equal(got[0][~bad], got[1][~bad])


@pytest.mark.parametrize("dtype,sizes", [("bf16", [0, 6, 10, 12, 14, 16, 20, 26, 40]), ("fp16", [0, 6, 10, 12, 13])])
@pytest.mark.parametrize("hq,hkv,new", [(8, 2, 300), (5, 1, 70), (4, 4, 129)])
def test_weights_of_logits_whose_terms_cancel(zc, dtype, sizes, hq, hkv, new):
    """Terms of up to 2^80 whose sums are small or rounding alone: under a window of one key every weight is 1, off by the
    log-sum-exp's rounding (2^-24 of it, a 20th where that is held to 1) and 2^-18; with two keys a row's sum to it."""
    dt, page, G = TYPES[dtype], 64, hq // hkv
    for size in sizes:
        gen = torch.Generator(device=DEV).manual_seed(7)
        table, n_pages = ref.make_table(np.random.RandomState(7), [new], page)
        k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
        q = torch.randn((new, hq, D), generator=gen, device=DEV).to(dt)
        k[..., 3:64] = (torch.randn((n_pages, page, hkv, 61), generator=gen, device=DEV) * 2.0 ** size).to(dt)
        q[..., 3:64] = (torch.randn((new, hq, 61), generator=gen, device=DEV) * 2.0 ** size).to(dt)
        k[..., 67:], q[..., 67:] = -k[..., 3:64], q[..., 3:64]
        pool = zc.PagedKV(k, v, hq, max_req=1, max_rows=new)
        for window in (1, 2):
            scores = torch.zeros((n_pages, hkv, page), device=DEV)
            out, lse = pool.attention_scored(q, i32(table), i32([0, new]), i32([new]), new, scores, window=window)
            settled(zc)
            mine = scores[torch.as_tensor(table[0], device=DEV).long()].transpose(1, 2).reshape(-1, hkv)[:new].double()
            assert torch.isfinite(mine).all() and mine.min() >= 0
            off = 2.0 ** (min(lse.abs().max().item(), 2.0 ** 20) * 2.0 ** -24) - 1 + 2.0 ** -18
            assert mine.max() <= window * G * (1 + off)
            if window == 1 and lse.abs().max() < 2.0 ** 20:
                assert mine.min() >= G * (1 - off)


# ---------------------------------------------------------------- pages that are none
def freed(table, n_pages, page, kv_len, lens, free, state):
    """The free list after the pages behind the kept tokens are put back, and its state; entries that are no page are not."""
    gone = [int(x) for r, (n, m) in enumerate(zip(kv_len, lens)) if m < n
            for x in table[r][-(-m // page): -(-n // page)] if 0 <= x < n_pages]
    free, nxt = list(free), min(max(state[0], 0), len(free))
    for i, p in enumerate(gone):
        if nxt - len(gone) + i >= 0:
            free[nxt - len(gone) + i] = p
    return free, [max(0, nxt - len(gone)), min(state[1], len(free)), max(0, len(gone) - nxt)]


@pytest.mark.parametrize("page,lengths,lens,room", [
    (16, [300, 17, 0, 40, 500], [128, 17, 0, 16, 0], 30), (64, [5000, 700], [1, 640], 200), (16, [160] * 300, [16] * 300, 3000),
    (16, [160] * 300, [16 * (i % 11) for i in range(300)], 700), (256, [4000], [0], 5), (16, [30000], [9000], 2000),
    (16, [20, 9000, 33], [4, 0, 0], 600), (16, [40] * 5000, [16 * (i % 3) for i in range(5000)], 9000),
    (16, [100000, 70], [16, 0], 7000)])
@pytest.mark.parametrize("holes", [0.0, 0.3, 1.0])
def test_only_pages_are_given_back(zc, page, lengths, lens, room, holes):
    rng, gen = np.random.RandomState(len(lengths)), torch.Generator(device=DEV).manual_seed(1)
    table, n_pages = ref.make_table(rng, lengths, page)
    table = table.copy()
    for r, m in enumerate(lens):
        behind = np.arange(table.shape[1]) >= -(-m // page)
        hole = behind & (rng.rand(table.shape[1]) < holes)
        table[r, hole] = rng.choice([-1, n_pages, 2 ** 31 - 1, -2 ** 31], size=int(hole.sum()))
    k, v = ref.make_pages(gen, n_pages, page, 1, torch.float16, False, DEV)
    pool = zc.PagedKV(k, v, 1, max_req=0, max_rows=0)
    most = max(1, max(lens))
    kept = i32(np.broadcast_to(np.arange(most), (len(lens), 1, most)).copy())
    free = rng.randint(0, 1000, room).tolist()
    state = [room - 2, room - 1, 5]
    dev = i32(free)
    out = pool.compact(i32(table), i32(lengths), kept, i32(lens), None, dev, i32(state))
    settled(zc)
    want, want_state = freed(table, n_pages, page, lengths, lens, free, state)
    assert dev.tolist() == want and out.tolist() == want_state


def test_thinning_out_where_the_pages_have_run_out(zc):
    """A step asks for more pages than are free; the requests are thinned out as they stand, and the next step's pages come
    from the list: every page is held once, and none is none."""
    page, hkv, n_pages, width = 16, 2, 24, 12
    gen = torch.Generator(device=DEV).manual_seed(3)
    k, v = ref.make_pages(gen, n_pages, page, hkv, torch.bfloat16, False, DEV)
    scores = torch.rand((n_pages, hkv, page), generator=gen, device=DEV)
    pool = zc.PagedKV(k, v, hkv, max_req=0, max_rows=0)
    free, table = i32(np.random.RandomState(1).permutation(n_pages)), torch.full((3, width), -1, dtype=torch.int32, device=DEV)
    one, two = zc.StepTables(3, 400), zc.StepTables(3, 400)
    one.build(page, i32([0, 0, 0]), i32([160, 100, 170]), free, i32([0, n_pages, 0]), table)
    settled(zc)
    assert one.free_state.tolist() == [n_pages, n_pages, 4] and (table[2, :11] == -1).sum() == 4
    keep = i32([64, 100, 60])
    kept, length = pool.select(table, one.kv_len, scores, keep, recent=8, first=i32([4, 4, 4]), max_keep=100)
    state = pool.compact(table, one.kv_len, kept, length, scores, free, one.free_state)
    settled(zc)
    assert length.tolist() == [64, 100, 60]
    back = (10 - 4) + (11 - 4 - 4)                   # request 2 held 7 of its 11 pages
    assert state.tolist() == [n_pages - back, n_pages, 0] and free.min() >= 0
    two.build(page, length, i32([48, 10, 40]), free, state, table)
    settled(zc)
    assert two.free_state.tolist()[2] == 0 and (two.slots[:98] >= 0).all()
    held = [int(x) for r, n in enumerate(two.kv_len.tolist()) for x in table[r, : -(-n // page)]]
    left = free[int(two.free_state[0]):].tolist()
    assert sorted(held + left) == list(range(n_pages))


# ---------------------------------------------------------------- budgets and lists
def test_a_request_within_its_budget_stays_whole_though_the_list_is_shorter(zc):
    """n <= keep[r] tokens stay, listed as far as the list goes; compaction leaves them; one token more is a selection."""
    page, hkv = 16, 2
    lengths, keep = [100, 100, 121, 120, 40, 41, 41], [100, 120, 120, 2 ** 31 - 1, 40, 41, 40]
    gen = torch.Generator(device=DEV).manual_seed(1)
    table, n_pages = ref.make_table(np.random.RandomState(1), lengths, page)
    k, v = ref.make_pages(gen, n_pages, page, hkv, torch.float16, False, DEV)
    scores = torch.rand((n_pages, hkv, page), generator=gen, device=DEV)
    pool = zc.PagedKV(k, v, hkv, max_req=0, max_rows=0)
    kept, length = pool.select(i32(table), i32(lengths), scores, i32(keep), 4, max_keep=40)
    settled(zc)
    assert length.tolist() == [100, 100, 40, 120, 40, 41, 40]
    for r in (0, 1, 3, 4, 5):
        assert (kept[r].cpu() == torch.arange(40)).all()
    for r in (2, 6):
        assert all((kept[r, h, 1:] > kept[r, h, :-1]).all() and kept[r, h, -4:].tolist() == list(range(lengths[r] - 4, lengths[r]))
                   for h in range(hkv))
    k2, v2, s2 = k.clone(), v.clone(), scores.clone()
    free = i32([0] * 30)
    state = pool.compact(i32(table), i32(lengths), kept, length, scores, free, i32([20, 30, 0]))
    settled(zc)
    assert state.tolist() == [20 - 5, 30, 0]              # 121 to 40 tokens: 8 pages to 3; 41 and 40 lie on three
    still = torch.as_tensor(np.unique(np.concatenate([table[r][: -(-lengths[r] // page)] for r in (0, 1, 3, 4, 5)])), device=DEV).long()
    assert torch.equal(k[still], k2[still]) and torch.equal(v[still], v2[still]) and torch.equal(scores[still], s2[still])


def test_a_selection_says_how_long_its_lists_are(zc):
    page, hkv = 16, 2
    table, n_pages = ref.make_table(np.random.RandomState(1), [100], page)
    k = torch.zeros((n_pages, page, hkv, D), dtype=torch.float16, device=DEV)
    scores = torch.zeros((n_pages, hkv, page), device=DEV)
    pool = zc.PagedKV(k, k, hkv, max_req=0, max_rows=0)
    args = (i32(table), i32([100]), scores, i32([20]))
    for bad in (dict(), dict(recent=8), dict(max_keep=-1)):
        with pytest.raises(zc.ZipCacheError, match="max_keep"):
            pool.select(*args, **bad)
    kept, length = pool.select(*args, kept=torch.empty((1, hkv, 20), dtype=torch.int32, device=DEV))
    settled(zc)
    assert length.tolist() == [20] and kept[0, 0].tolist() == list(range(20))
    kept, length = pool.select(*args, max_keep=0)          # said so: nothing is kept
    settled(zc)
    assert kept.shape == (1, hkv, 0) and length.tolist() == [0]


# ---------------------------------------------------------------- slots that two requests score
@pytest.mark.parametrize("new", [1, 40])
def test_slots_that_two_requests_score_hold_some_number_and_others_their_own(zc, new):
    """Pages that requests share belong before `first`.  Where they do not, their slots end with a number of 0 to what the
    requests' rows could add to the old score; every other slot is as if nothing were shared."""
    hq, hkv, page, shared = 8, 2, 16, 160
    rng, gen, dt = np.random.RandomState(5), torch.Generator(device=DEV).manual_seed(6), torch.bfloat16
    table, kv, starts, n_pages, copies = er.make_groups(rng, page, [4], [shared], [new + 40, new + 3, new, new + 100])
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
    q = torch.randn(4 * new, hq, D, generator=gen, device=DEV).to(dt)
    row_start = [new * i for i in range(5)]
    pool = zc.PagedKV(k, v, hq, max_req=4, max_rows=4 * new, scored_rows=1)
    start = torch.rand((n_pages, hkv, page), generator=gen, device=DEV)
    got, want = start.clone(), start.clone()
    pool.attention_scored(q, i32(table), i32(row_start), i32(kv), new, got)
    pool.attention_scored(q, i32(table), i32(row_start), i32(kv), new, want, first=i32([shared] * 4))
    settled(zc)
    common = torch.zeros(n_pages, dtype=torch.bool, device=DEV)
    common[torch.as_tensor(table[0, : shared // page], device=DEV).long()] = True
    assert torch.equal(got[~common], want[~common]) and torch.equal(want[common], start[common])
    more = (got - start)[common]
    # (an old score and its sum are off by half a step each)
    assert more.min() >= -2.0 ** -22 and more.max() <= new * hq // hkv * (1 + 2.0 ** -22)


def test_own_tokens_of_a_group_that_shares_more_than_it_says(zc):
    """said < what the tables share, with scores: outputs are right, and the scores of the slots that are one request's."""
    hq, hkv, page = 8, 2, 16
    rng, gen, dt = np.random.RandomState(8), torch.Generator(device=DEV).manual_seed(9), torch.float16
    table, kv, starts, n_pages, copies = er.make_groups(rng, page, [8], [960], [30 + i for i in range(8)])
    common = torch.as_tensor(table[0, :60], device=DEV).long()
    table = wide(table, page, hkv, 1)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
    q = torch.randn(8, hq, D, generator=gen, device=DEV).to(dt)
    pool = zc.PagedKV(k, v, hq, max_req=8, max_rows=8, shared=True, scored_rows=1)
    start = torch.rand((n_pages, hkv, page), generator=gen, device=DEV)
    got = start.clone()
    out, lse = pool.attention_shared(q, i32(table), i32(range(9)), i32(kv), 1, i32(starts), i32([800]), scores=got)
    settled(zc)
    want, tol = er.add_weights(start, q, k, table, list(range(9)), kv, [960] * 8, 0, 0)
    alone = torch.ones(n_pages, dtype=torch.bool, device=DEV)
    alone[common] = False
    assert ((got.double() - want).abs() <= tol)[alone].all()
    assert torch.equal(got[common[:50]], start[common[:50]])             # what the call was told is shared has no score
    more = (got - start)[common[50:]]
    assert more.min() >= -2.0 ** -22 and more.max() <= hq // hkv * (1 + 2.0 ** -22)


@pytest.mark.parametrize("per", range(1, 17))
def test_every_number_of_logits_to_a_key(zc, per):
    """Query heads of a KV head times rows, all that single tokens' kernels take."""
    hkv, page = 2, 16
    for G in (g for g in range(1, per + 1) if per % g == 0):
        most, gen, dt = per // G, torch.Generator(device=DEV).manual_seed(per), torch.float16
        new = [most, 1, max(1, most - 1)]
        kv = [n + p for n, p in zip(new, (70, 0, 301))]
        table, n_pages = ref.make_table(np.random.RandomState(per), kv, page)
        k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
        row_start = [0] + np.cumsum(new).tolist()
        q = torch.randn(row_start[-1], hkv * G, D, generator=gen, device=DEV).to(dt)
        pool = zc.PagedKV(k, v, hkv * G, max_req=3, max_rows=row_start[-1], scored_rows=most)
        start = torch.rand((n_pages, hkv, page), generator=gen, device=DEV)
        got = start.clone()
        pool.attention_scored(q, i32(table), i32(row_start), i32(kv), most, got, first=i32([3, 0, 0]))
        settled(zc)
        want, tol = er.add_weights(start, q, k, table, row_start, kv, [3, 0, 0], 0, 0)
        assert ((got.double() - want).abs() <= tol).all()


def test_compaction_of_no_requests_says_the_free_list_s_state(zc):
    k = torch.zeros((4, 16, 2, D), dtype=torch.float16, device=DEV)
    pool = zc.PagedKV(k, k, 2, max_req=0, max_rows=0)
    none, table = i32([]), torch.zeros((0, 5), dtype=torch.int32, device=DEV)
    kept = torch.zeros((0, 2, 8), dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    for given, state, want in ((None, [2, 4, 7], [2, 4, 0]), (i32([9, 9, 9]), [-3, 9, 1], [0, 4, 0]), (None, [6, 4, 0], [4, 4, 0])):
        torch.full((3,), 77, dtype=torch.int32, device=DEV)          # (freed: what an unwritten result would hold)
        for stream in (None, side):
            out = pool.compact(table, none, kept, none, None, i32([0, 1, 2, 3]), i32(state), given, stream=stream)
            settled(zc)
            assert out.tolist() == want and (given is None or out is given)
    assert pool.compact(table, none, kept, none) is None
