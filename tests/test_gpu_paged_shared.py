"""Attention of requests that begin alike, on the GPU, against 64 bits under the bounds derived in zc_paged_ref; and the
run of it all: a shared prompt, generated tokens that are weighed, the selection, the compaction, and on."""
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


def widened(table, page, hkv, n_groups):
    """The table with so many more (empty) columns that sharing may pay by its width: calls that cannot save 90 MB of reads
    are attended like any."""
    spare = len(table) - min(n_groups, len(table))
    width = int(1e8 / max(1, spare * hkv * 512 * page)) + 1
    return np.pad(table, ((0, 0), (0, max(0, width - table.shape[1]))), constant_values=-1)


def check_rows(dt, q, k, v, table, row_start, kv, out, lse):
    hq, hkv = q.shape[1], k.shape[2]
    vmax = v.abs().max().double()
    for r, n in enumerate(kv):
        a, e = row_start[r], row_start[r + 1]
        if a == e:
            continue
        kr, vr = ref.rows_of_request(k, v, table[r], n)
        for h in range(hq):
            o, l, mean_abs, largest, seen, total = ref.attend(q[a:e, h], kr[:, h // (hq // hkv)], vr[:, h // (hq // hkv)],
                                                              n - (e - a), 0, 0)
            t_out, t_lse = ref.tolerances(dt, o, mean_abs, largest, seen, total, vmax)
            some = seen > 0
            bad = ((out[a:e, h].double() - o).abs() - t_out)[some]
            assert torch.isfinite(out[a:e, h]).all() and (bad.numel() == 0 or bad.max() <= 0), (r, h, bad.max().item())
            off = ((lse[a:e, h].double() - l).abs() - t_lse)[some]
            assert off.numel() == 0 or off.max() <= 0, (r, h, off.max().item())
            assert (out[a:e, h][~some] == 0).all() and (lse[a:e, h][~some] == -math.inf).all()


def shared_case(zc, dtype, hq, hkv, page, groups, shared, own, new=1, alone=0, heads_first=False, pad_rows=0, scored=False,
                said=None, kv_len=None, seed=0, wide=True):
    """groups requests with these shared lengths and own lengths behind them (new tokens included); said: what the caller
    claims to be shared, where that is another number."""
    rng, gen, dt = np.random.RandomState(seed), torch.Generator(device=DEV).manual_seed(seed + 1), TYPES[dtype]
    table, kv, starts, n_pages, copies = er.make_groups(rng, page, groups, shared, own, alone)
    if wide:
        table = widened(table, page, hkv, len(groups))
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, heads_first, DEV)
    for src, dst, rows in copies:
        for pool in (k, v):
            pool[dst, :rows] = pool[src, :rows]
    if kv_len is not None:
        kv = kv_len
    new = [new] * len(kv) if isinstance(new, int) else new
    row_start = [0] + np.cumsum(new).tolist()
    rows = row_start[-1] + pad_rows
    q = torch.randn(rows, hq, D, generator=gen, device=DEV).to(dt)
    if pad_rows:
        q[row_start[-1]:] = math.nan
    # what no request has is NaN
    held = torch.zeros((n_pages, page), dtype=torch.bool, device=DEV)
    for r, n in enumerate(kv):
        t = torch.arange(n, device=DEV)
        held[torch.as_tensor(table[r], device=DEV).long()[t // page], t % page] = True
    ck, cv = k.clone(), v.clone()
    for pool in (k, v):
        pool[~held] = math.nan
    pool = zc.PagedKV(k, v, hq, max_req=len(kv), max_rows=rows, shared=True, scored_rows=max(new) if scored else 0)
    pool.workspace[zc.ZC_PAGES_SYNC_BYTES:] = 0xFF
    out = torch.full((rows, hq, D), 9.0, dtype=dt, device=DEV)
    lse = torch.full((rows, hq), 9.0, device=DEV)
    scores = torch.rand((n_pages, hkv, page), generator=gen, device=DEV) if scored else None
    before = scores.clone() if scored else None
    said = shared if said is None else said
    args = (q, i32(table), i32(row_start), i32(kv), max(max(new), 1), i32(starts), i32(said))
    pool.attention_shared(*args, scores=scores, out=out, row_lse=lse)
    settled(zc)
    check_rows(dt, q, ck, cv, table, row_start, kv, out, lse)
    assert (out[row_start[-1]:] == 9).all() and (lse[row_start[-1]:] == 9).all()
    assert (pool.workspace[:zc.ZC_PAGES_SYNC_BYTES] == 0).all()
    if scored:
        first = [0] * len(kv)
        for g, s in enumerate(said):
            first[starts[g]:starts[g + 1]] = [max(0, s)] * (starts[g + 1] - starts[g])
        want, tol = er.add_weights(before, q, ck, table, row_start, kv, first, 0, 0)
        bad = (scores.double() - want).abs() - tol
        assert bad.max() <= 0, bad.max().item()
        assert torch.equal(scores[tol == 0], before[tol == 0])
    return pool, args, out, lse


CASES = [
    dict(hq=8, hkv=2, page=16, groups=[3], shared=[1000], own=[1, 40, 300]),
    dict(hq=32, hkv=8, page=64, groups=[20], shared=[2048], own=[1 + 13 * i for i in range(20)]),          # 80 rows
    dict(hq=32, hkv=8, page=64, groups=[70], shared=[1500], own=[1 + i for i in range(70)]),               # 280 rows: two items
    dict(hq=4, hkv=4, page=32, groups=[5, 2, 9], shared=[700, 64, 333], own=list(range(1, 17))),           # G = 1
    dict(hq=6, hkv=2, page=256, groups=[50], shared=[600], own=[5] * 50, heads_first=True),                # G = 3
    dict(hq=16, hkv=1, page=16, groups=[30], shared=[5000], own=[9] * 30),                                 # one head, G = 16
    dict(hq=8, hkv=2, page=16, groups=[4, 3], shared=[900, 130], own=[7] * 10, alone=3, pad_rows=4),       # requests in no group
    dict(hq=8, hkv=2, page=16, groups=[4], shared=[900], own=[7, 9, 30, 4], new=[4, 1, 3, 2]),             # a few tokens each
    dict(hq=2, hkv=2, page=16, groups=[6], shared=[800], own=[20, 30, 17, 18, 40, 16], new=[16, 9, 0, 3, 16, 1]),
    dict(hq=8, hkv=2, page=16, groups=[1, 5], shared=[4000, 2000], own=[3] * 6),                           # a group of one
    dict(hq=8, hkv=2, page=16, groups=[0, 5, 0], shared=[300, 2000, 40], own=[3] * 5),                     # groups of none
    dict(hq=8, hkv=2, page=16, groups=[3], shared=[10], own=[60, 1, 5]),                                   # too short to share
    dict(hq=8, hkv=2, page=16, groups=[5], shared=[0], own=[60, 1, 5, 300, 7]),
    dict(hq=8, hkv=2, page=64, groups=[8], shared=[640], own=[1] * 8, said=[640 + 500]),                   # more than there is
    dict(hq=8, hkv=2, page=64, groups=[8], shared=[640], own=[5] * 8, said=[-3]),
    dict(hq=8, hkv=2, page=64, groups=[8], shared=[640], own=[5] * 8, said=[2 ** 31 - 1]),
    dict(hq=8, hkv=2, page=64, groups=[8], shared=[640], own=[5] * 8, said=[100]),                         # less
    dict(hq=8, hkv=2, page=16, groups=[2] * 60, shared=[400 + i for i in range(60)], own=[3] * 120),       # many groups
    dict(hq=8, hkv=8, page=64, groups=[130], shared=[200], own=[3] * 130),
    dict(hq=4, hkv=2, page=16, groups=[4], shared=[600], own=[1] * 4, new=[4, 3, 2, 1], kv_len=[2, 601, 601, 601]),   # rows that see nothing
    dict(hq=7, hkv=1, page=16, groups=[19], shared=[900], own=[5 + i for i in range(19)]),                 # G = 7: 126 of 128 rows
    dict(hq=10, hkv=2, page=128, groups=[6, 30], shared=[3000, 129], own=[200] * 36, new=[3, 1, 2] * 12),  # G = 5, 15 rows
]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("kw", CASES)
def test_groups(zc, dtype, kw):
    shared_case(zc, dtype, **kw)


@pytest.mark.parametrize("kw", [CASES[0], CASES[6], CASES[7]])
def test_groups_that_cannot_save_much(zc, kw):
    """Narrow tables: attended like any, by one kernel."""
    shared_case(zc, "bf16", scored=True, wide=False, **kw)
    pool, args, out, lse = shared_case(zc, "fp16", wide=False, **kw)
    o, l = pool.attention(*args[:5])
    settled(zc)
    end = int(args[2][-1])
    assert torch.equal(out[:end], o[:end]) and torch.equal(lse[:end], l[:end])
    before = zc.zc_pages_launch_count(pool.handle)
    pool.attention_shared(*args)
    assert zc.zc_pages_launch_count(pool.handle) == before + 1
    settled(zc)


def test_own_parts_of_every_length(zc):
    """Pieces of the own keys: from one block to more than there is room for at the shortest, more than a warp's batch."""
    shared_case(zc, "fp16", 8, 2, 64, groups=[5], shared=[512], own=[30000, 1, 16, 17, 64])
    shared_case(zc, "bf16", 4, 4, 16, groups=[40], shared=[512], own=[1 + 37 * i for i in range(40)], seed=3)
    shared_case(zc, "fp16", 2, 1, 16, groups=[900], shared=[640], own=[1 + i % 130 for i in range(900)], seed=4)     # > kPlanReq requests
    shared_case(zc, "fp16", 32, 32, 16, groups=[9, 9], shared=[700, 64], own=[500] * 18, seed=5)


def test_more_pieces_than_a_warp_knows_at_once(zc):
    """Long shared keys leave few SMs to 4160 short own parts: some 35 to each of their warps, which know 32 at a time."""
    shared_case(zc, "fp16", 32, 32, 64, groups=[130], shared=[66000], own=[1 + i % 40 for i in range(130)], seed=6)


@pytest.mark.parametrize("kw", [CASES[0], CASES[2], CASES[3], CASES[6], CASES[7], CASES[13], CASES[11]])
def test_groups_with_scores(zc, kw):
    shared_case(zc, "bf16", scored=True, **kw)


def test_calls_repeat_bit_for_bit_and_serve_other_calls(zc):
    """One workspace for shared calls and plain ones of every kind, in turn; captured and replayed with other lengths."""
    pool, args, out, lse = shared_case(zc, "fp16", 8, 2, 16, [6, 4], [1500, 300], [40] * 10)
    q, table, row_start, kv, most, starts, said = args
    kv2 = kv.clone()
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    for _ in range(3):
        pool.attention(q, table, row_start, kv, 1)
        pool.attention(q, table, i32([0, 10] + [10] * 9), kv, 10)          # a chunk
        pool.attention_shared(*args, out=o2, row_lse=l2)
        settled(zc)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pool.attention_shared(q, table, row_start, kv2, most, starts, said, out=o2, row_lse=l2)
    for cut in (0, 7, 39, 300):
        kv2.copy_(kv - cut)
        graph.replay()
        settled(zc)
        want = pool.attention_shared(q, table, row_start, kv - cut, most, starts, said)
        settled(zc)
        assert torch.equal(want[0], o2) and torch.equal(want[1], l2)
    check_rows(torch.float16, q, *(torch.nan_to_num(t) for t in (pool.k_pages, pool.v_pages)), table.cpu().numpy(),
               row_start.tolist(), kv2.tolist(), o2, l2)


def test_more_rows_than_the_bound_and_lengths_beyond_the_table(zc):
    """A request with more rows than the caller vouched for does not disturb the others, nor does one whose length passes
    the table's end."""
    hq, hkv, page = 8, 2, 16
    rng, gen = np.random.RandomState(5), torch.Generator(device=DEV).manual_seed(6)
    table, kv, starts, n_pages, copies = er.make_groups(rng, page, [5], [800], [40, 30, 64, 50, 20])
    table = widened(table, page, hkv, 1)
    k, v = ref.make_pages(gen, n_pages, page, hkv, torch.bfloat16, False, DEV)
    new = [1, 2, 5, 1, 2]
    row_start = [0] + np.cumsum(new).tolist()
    q = torch.randn(row_start[-1], hq, D, generator=gen, device=DEV).to(torch.bfloat16)
    scores = torch.zeros((n_pages, hkv, page), device=DEV)
    pool = zc.PagedKV(k, v, hq, max_req=5, max_rows=row_start[-1], shared=True, scored_rows=2)
    out, lse = pool.attention_shared(q, i32(table), i32(row_start), i32(kv), 2, i32(starts), i32([800]), scores=scores)
    settled(zc)
    ok = [0, 1, 3, 4]
    check_rows(torch.bfloat16, q, k, v, table, [row_start[r] for r in range(6)], [kv[r] if r in ok else 0 for r in range(5)],
               out.index_fill(0, torch.arange(3, 8, device=DEV), 0.0), lse.index_fill(0, torch.arange(3, 8, device=DEV), -math.inf))
    assert torch.isfinite(scores).all()
    narrow = i32(table[:, :53].copy())           # 848 tokens: 840 and 864 are requests 0 and 2
    pool.attention_shared(q, narrow, i32(row_start), i32([2 ** 30, 830, 900, 850, 820]), 2, i32(starts), i32([800]), scores=scores)
    settled(zc)


def test_streams_and_no_groups_with_scores(zc):
    pool, args, out, lse = shared_case(zc, "bf16", 8, 2, 64, [6], [2000], [40] * 6, scored=True)
    q, table, row_start, kv, most, starts, said = args
    side = torch.cuda.Stream()
    scores = torch.zeros(pool.k_pages.shape[0], 2, 64, device=DEV)
    torch.cuda.synchronize()
    torch.cuda._sleep(int(2e7))
    o, l = pool.attention_shared(*args, scores=scores, stream=side)
    side.synchronize()
    assert torch.equal(o, out) and torch.equal(l, lse)
    kept, length = pool.select(table, kv, scores, i32([2010] * 6), 4, first=i32([2000] * 6), max_keep=2010, stream=side)
    free, state = i32([0] * 50), i32([40, 50, 0])
    after = pool.compact(table, kv, kept, length, scores, free, state, stream=side)
    side.synchronize()
    assert length.tolist() == [2010] * 6 and after.tolist() == [40, 50, 0]      # (the last page holds 2010 and 2040 alike)
    one, two = torch.zeros_like(scores), torch.zeros_like(scores)
    pool.attention_shared(q, table, row_start, kv, 1, i32([0]), i32([]), scores=one)
    pool.attention_scored(q, table, row_start, kv, 1, two)
    settled(zc)
    own = table[:, 31].long()                    # (a slot that several requests score ends with one's sum)
    assert torch.equal(one[own], two[own]) and one[own].max() > 0


def test_no_groups_and_borders_that_contradict(zc):
    pool, args, out, lse = shared_case(zc, "bf16", 8, 2, 16, [6, 4], [1500, 300], [40] * 10)
    q, table, row_start, kv, most, starts, said = args
    plain, plain_lse = pool.attention(q, table, row_start, kv, 1)
    none, none_lse = pool.attention_shared(q, table, row_start, kv, 1, i32([0]), i32([]))
    settled(zc)
    assert torch.equal(plain, none) and torch.equal(plain_lse, none_lse)
    for bad in ([0, 9, 2], [-5, 3, 100], [7, 7, 7], [2 ** 31 - 1, -2 ** 31, 4]):      # no fault; what comes out is not said
        pool.attention_shared(q, table, row_start, kv, 1, i32(bad), said)
    pool.attention_shared(q, table, i32([0, 9, 3, 12, -4, 2, 8, 1, 90, 5, 10]), kv, 1, i32([0, 10] * 30 + [0]), i32([900] * 60))
    settled(zc)
    again, again_lse = pool.attention_shared(*args)
    settled(zc)
    assert torch.equal(again, out) and torch.equal(again_lse, lse)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
def test_maxima_far_apart_between_shared_and_own_keys(zc, dtype):
    """The shared keys far above the own ones, and far below: the join drops what weighs nothing and keeps the rest."""
    for loud_own in (False, True):
        rng, gen, dt = np.random.RandomState(1), torch.Generator(device=DEV).manual_seed(2), TYPES[dtype]
        table, kv, starts, n_pages, copies = er.make_groups(rng, 16, [4], [640], [30, 31, 1, 200])
        table = widened(table, 16, 2, 1)
        k, v = ref.make_pages(gen, n_pages, 16, 2, dt, False, DEV)
        own_pages = torch.as_tensor(np.unique(table[:, 40:][table[:, 40:] >= 0]), device=DEV).long()
        shared_pages = torch.as_tensor(np.unique(table[:, :40]), device=DEV).long()
        k[own_pages if loud_own else shared_pages] *= 16.0
        q = (torch.randn(4, 8, D, generator=gen, device=DEV) * 4).to(dt)
        pool = zc.PagedKV(k, v, 8, max_req=4, max_rows=4, shared=True)
        out, lse = pool.attention_shared(q, i32(table), i32([0, 1, 2, 3, 4]), i32(kv), 1, i32(starts), i32([640]))
        settled(zc)
        check_rows(dt, q, k, v, table, [0, 1, 2, 3, 4], kv, out, lse)


def test_a_run_of_it_all(zc):
    """Two prompts with four and three conversations, tables by the step's own plan, every token weighed; when the
    conversations are over their budget, what they keep is selected and moved, pages come back, and the next tokens go on
    over the thinned-out cache.  Checked against plain attention over the rows that a Python bookkeeping says are there."""
    page, hq, hkv, dt = 16, 8, 2, torch.bfloat16
    gen = torch.Generator(device=DEV).manual_seed(11)
    shared, groups = [320, 96], [4, 3]
    starts, n_req = [0, 4, 7], 7
    n_pages, width = 260, 1300
    k = torch.full((n_pages, page, hkv, D), math.nan, dtype=dt, device=DEV)
    v = k.clone()
    scores = torch.full((n_pages, hkv, page), math.nan, device=DEV)
    pool = zc.PagedKV(k, v, hq, max_req=n_req, max_rows=n_req, shared=True, scored_rows=1)
    free, table = i32(np.random.RandomState(0).permutation(n_pages)), torch.full((n_req, width), -1, dtype=torch.int32, device=DEV)
    steps = [zc.StepTables(n_req, n_req), zc.StepTables(n_req, n_req)]
    # the prompts' pages: taken by hand, the same for all of a group (whole pages)
    state, at = i32([0, n_pages, 0]), 0
    rows = torch.randn(2, sum(shared), hkv, D, generator=gen, device=DEV).to(dt)
    ids = free.tolist()
    mem = [[] for _ in range(n_req)]          # per request: [head] lists of (key, value)
    off = 0
    for g, s in enumerate(shared):
        pages = ids[at:at + s // page]
        at += s // page
        for r in range(starts[g], starts[g + 1]):
            table[r, : s // page] = i32(pages)
            mem[r] = [[(rows[0, off + t, h], rows[1, off + t, h]) for t in range(s)] for h in range(hkv)]
        slots = [pages[t // page] * page + t % page for t in range(s)]
        pool.write(rows[0, off:off + s], rows[1, off:off + s], i32(slots))
        off += s
    state = i32([at, n_pages, 0])
    past = i32([s for s, n in zip(shared, groups) for _ in range(n)])
    first = past.clone()
    one, row_start = i32([1] * n_req), list(range(n_req + 1))
    for step in range(75):
        plan = steps[step % 2].build(page, past, one, free, state, table)
        new = torch.randn(2, n_req, hkv, D, generator=gen, device=DEV).to(dt)
        q = torch.randn(n_req, hq, D, generator=gen, device=DEV).to(dt)
        pool.write(new[0], new[1], plan.slots)
        out, lse = pool.attention_shared(q, table, plan.row_start, plan.kv_len, 1, i32(starts), i32(shared), scores=scores)
        for r in range(n_req):
            for h in range(hkv):
                mem[r][h].append((new[0, r, h], new[1, r, h]))
        state, past = plan.free_state, plan.kv_len
        if step in (0, 39, 40, 74):
            settled(zc)
            for r in range(n_req):
                for h in range(hq):
                    kr, vr = (torch.stack([x[i] for x in mem[r][h // 4]]) for i in (0, 1))
                    assert past[r] == len(mem[r][0])
                    o, l, mean_abs, largest, seen, total = ref.attend(q[r:r + 1, h], kr, vr, kr.shape[0] - 1, 0, 0)
                    t_out, t_lse = ref.tolerances(dt, o, mean_abs, largest, seen, total, 10.0)
                    assert ((out[r:r + 1, h].double() - o).abs() <= t_out).all()
                    assert ((lse[r:r + 1, h].double() - l).abs() <= t_lse).all()
        if step == 39:
            was = state.tolist()
            keep = first + i32([17, 40, 9, 100, 16, 33, 24])
            kept, length = pool.select(table, past, scores, keep, recent=8, first=first, max_keep=int(keep.max()))
            state = pool.compact(table, past, kept, length, scores, free, state)
            settled(zc)
            for r in range(n_req):
                m = int(length[r])
                assert m == min(int(past[r]), int(keep[r]))
                for h in range(hkv):
                    pos = kept[r, h, :m].tolist()
                    assert pos[: int(first[r])] == list(range(int(first[r]))) and pos[-8:] == list(range(int(past[r]) - 8, int(past[r])))
                    mem[r][h] = [mem[r][h][i] for i in pos]
            back = sum(-(-int(a) // page) + (-int(b) // page) for a, b in zip(past, length))
            assert back > 0 and state.tolist() == [was[0] - back, n_pages, 0]
            past = length
            # (scores of a step's own tokens start anew in the pages that come back)
    live = torch.zeros((n_pages, page), dtype=torch.bool, device=DEV)
    for r in range(n_req):
        t = torch.arange(int(first[r]), int(past[r]), device=DEV)
        live[table[r].long()[t // page], t % page] = True
    assert torch.isfinite(scores.transpose(1, 2)[live]).all() and scores.transpose(1, 2)[live].min() >= 0
