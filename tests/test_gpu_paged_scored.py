"""Attention that adds up the cached tokens' weights, on the GPU: outputs bit for bit those of the attention beside it,
scores against 64 bits under the bounds derived in zc_evict_ref."""
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


def scored_case(zc, dtype, hq, hkv, page, past, new, window=0, sinks=0, first=None, heads_first=False, strided=False,
                pad_rows=0, kv_len=None, seed=0):
    """Every place that no row of the call sees holds NaN, in scores as in keys; the slots' old scores and NaN around them
    stay as they were, bit for bit, where no row sees them."""
    rng, gen, dt = np.random.RandomState(seed), torch.Generator(device=DEV).manual_seed(seed + 1), TYPES[dtype]
    kv = [p + n for p, n in zip(past, new)] if kv_len is None else kv_len
    first = [0] * len(kv) if first is None else first
    table, n_pages = ref.make_table(rng, kv, page)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, heads_first, DEV)
    row_start = [0] + np.cumsum(new).tolist()
    rows = row_start[-1] + pad_rows
    joint = torch.randn(rows, hq + (2 * hkv if strided else 0), D, generator=gen, device=DEV).to(dt)
    q = joint[:, :hq]
    if pad_rows:
        joint[row_start[-1]:] = math.nan
    scores = torch.rand((n_pages, hkv, page), generator=gen, device=DEV) * 3
    clean = k.clone()
    live = torch.zeros((n_pages, page), dtype=torch.bool, device=DEV)
    fresh = torch.zeros_like(live)
    for r, n in enumerate(kv):
        p0 = n - new[r]
        t = torch.arange(n, device=DEV)
        lo = max(0, p0 - window + 1) if window else 0
        seen = ((t >= lo) | (t < sinks)) if new[r] else torch.zeros_like(t, dtype=torch.bool)
        at = (torch.as_tensor(table[r], device=DEV).long()[t // page], t % page) if n else None
        if n:
            live[at] = seen
            fresh[at] = (t >= p0) & (t >= first[r])
    for pool in (k, v):
        pool[~live] = math.nan
    scores.transpose(1, 2)[fresh & live] = math.nan       # a new token's slot may hold anything
    before = scores.clone()
    few = max(new) * (hq // hkv) <= 16
    pool = zc.PagedKV(k, v, hq, max_req=len(kv), max_rows=rows, scored_rows=max(new) if few else 0)
    if pool.logits is not None:
        pool.logits.fill_(0xFF)                           # NaN
    out, lse = (torch.full(s, 9.0, dtype=t, device=DEV) for s, t in (((rows, hq, D), dt), ((rows, hq), torch.float32)))
    args = (q, i32(table), i32(row_start), i32(kv), max(max(new), 1))
    pool.attention_scored(*args, scores, first=i32(first), window=window, sinks=sinks, out=out, row_lse=lse)
    settled(zc)
    o2, l2 = torch.full_like(out, 9.0), torch.full_like(lse, 9.0)
    pool.attention(*args, window=window, sinks=sinks, out=o2, row_lse=l2)
    settled(zc)
    assert torch.equal(out.view(torch.int16), o2.view(torch.int16)) and torch.equal(lse, l2)
    want, tol = er.add_weights(torch.nan_to_num(before, nan=0.0), q, clean, table, row_start, kv, first, window, sinks)
    touched = torch.zeros_like(live)
    for r, n in enumerate(kv):
        t = torch.arange(n, device=DEV)
        if n and new[r]:
            at = (torch.as_tensor(table[r], device=DEV).long()[t // page], t % page)
            touched[at] = live[at] & (t >= first[r])
    m = touched[:, None].expand_as(scores)
    assert torch.equal(scores[~m].view(torch.int32), before[~m].view(torch.int32))
    assert torch.isfinite(scores[m]).all()
    bad = ((scores.double() - want).abs() - tol)[m]
    assert bad.numel() == 0 or bad.max() <= 0, (bad.max().item(), tol[m].max().item())
    return pool, args, scores, before


FEW = [
    dict(hq=1, hkv=1, page=16, past=[0], new=[1]),
    dict(hq=4, hkv=4, page=16, past=[15, 16, 17, 127, 128, 129], new=[1] * 6, first=[0, 16, 5, 128, 4, 1000]),
    dict(hq=32, hkv=8, page=64, past=[200, 511, 1, 0], new=[1] * 4, strided=True, first=[4] * 4),
    dict(hq=8, hkv=1, page=128, past=[5000], new=[1]),
    dict(hq=16, hkv=1, page=32, past=[777, 3], new=[1, 1]),
    dict(hq=6, hkv=2, page=256, past=[1000, 256, 255], new=[1, 1, 1], heads_first=True),
    dict(hq=14, hkv=2, page=16, past=[300, 40], new=[1, 1]),
    dict(hq=9, hkv=1, page=16, past=[300, 40], new=[1, 1]),
    dict(hq=32, hkv=32, page=64, past=[100, 900, 2048], new=[1] * 3),
    dict(hq=8, hkv=2, page=16, past=[60, 900, 3], new=[4, 3, 2], first=[0, 901, 4]),
    dict(hq=2, hkv=2, page=16, past=[70, 0, 200], new=[16, 9, 0]),
    dict(hq=4, hkv=2, page=64, past=[10, 20, 30], new=[1, 0, 1], pad_rows=5),
    dict(hq=4, hkv=1, page=16, past=[0] * 4, new=[1] * 4, kv_len=[0, 1, 0, 30]),
    dict(hq=4, hkv=2, page=16, past=[0] * 3, new=[4, 3, 2], kv_len=[2, 0, 2]),
    dict(hq=8, hkv=2, page=16, past=[i * 7 % 390 for i in range(300)], new=[i % 2 for i in range(300)]),
]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("kw", FEW)
def test_single_tokens_and_few_rows(zc, dtype, kw):
    scored_case(zc, dtype, **kw)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (16, 0), (33, 4), (128, 128), (500, 1), (2 ** 31 - 1, 2 ** 31 - 1)])
def test_single_tokens_under_a_window(zc, window, sinks):
    scored_case(zc, "fp16", 8, 2, 16, [0, 15, 90, 130, 640, 1500], [1, 1, 2, 1, 4, 1], window=window, sinks=sinks)
    scored_case(zc, "bf16", 4, 4, 64, [33, 700, 2047], [1, 1, 1], window=window, sinks=sinks, first=[0, 3, 2000])


CHUNK = [
    dict(hq=4, hkv=1, page=16, past=[0], new=[5]),
    dict(hq=1, hkv=1, page=16, past=[0, 3], new=[17, 300]),
    dict(hq=32, hkv=8, page=64, past=[0, 100, 700], new=[64, 1, 65], strided=True, first=[4, 4, 710]),
    dict(hq=8, hkv=2, page=128, past=[1000, 0, 5], new=[130, 0, 257], heads_first=True),
    dict(hq=6, hkv=2, page=32, past=[77, 300], new=[100, 43]),
    dict(hq=5, hkv=1, page=256, past=[500, 0], new=[60, 300], first=[513, 0]),
    dict(hq=16, hkv=1, page=16, past=[129, 31], new=[20, 8]),
    dict(hq=14, hkv=2, page=16, past=[129, 31], new=[40, 8], pad_rows=9),
    dict(hq=4, hkv=4, page=64, past=[3000], new=[33]),
    dict(hq=8, hkv=1, page=16, past=[4000, 20], new=[100, 3]),
    dict(hq=8, hkv=8, page=16, past=[10, 0, 128, 127, 1], new=[256, 128, 127, 129, 40]),
    dict(hq=4, hkv=2, page=16, past=[0] * 4, new=[40, 30, 20, 33], kv_len=[13, 0, 20, 1]),
    dict(hq=8, hkv=2, page=16, past=[i * 3 % 90 for i in range(150)], new=[(i * 5) % 21 for i in range(150)]),
    dict(hq=2, hkv=2, page=64, past=[0], new=[1500]),
]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("kw", CHUNK)
def test_chunks(zc, dtype, kw):
    scored_case(zc, dtype, **kw)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (31, 0), (64, 4), (128, 128), (200, 130), (600, 300)])
def test_chunks_under_a_window(zc, window, sinks):
    scored_case(zc, "fp16", 8, 2, 16, [0, 90, 1000, 130], [150, 33, 70, 1], window=window, sinks=sinks)
    scored_case(zc, "bf16", 2, 2, 128, [700, 2000], [300, 140], window=window, sinks=sinks, first=[0, 64])


def test_scores_add_up_over_steps_and_do_not_depend_on_timing(zc):
    """A prompt in a chunk, then tokens one by one, twice over: the same bits; every row's weights sum to 1, so a request's
    scores of a KV head sum to its rows times the query heads of the head."""
    hq, hkv, page, dt = 8, 2, 16, torch.bfloat16
    gen = torch.Generator(device=DEV).manual_seed(4)
    n0, steps = [70, 3, 200], 5
    table, n_pages = ref.make_table(np.random.RandomState(4), [n + steps for n in n0], page)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
    q = torch.randn(sum(n0) + 3 * steps, hq, D, generator=gen, device=DEV).to(dt)
    pool = zc.PagedKV(k, v, hq, max_req=3, max_rows=300, scored_rows=1)
    got = []
    for _ in range(2):
        scores = torch.full((n_pages, hkv, page), math.nan, device=DEV)
        pool.attention_scored(q[:sum(n0)], i32(table), i32([0, 70, 73, 273]), i32(n0), 200, scores)
        for s in range(steps):
            at = sum(n0) + 3 * s
            pool.attention_scored(q[at:at + 3], i32(table), i32([0, 1, 2, 3]), i32([n + s + 1 for n in n0]), 1, scores)
        settled(zc)
        got.append(scores)
    assert torch.equal(got[0].view(torch.int32), got[1].view(torch.int32))
    for r, n in enumerate(n0):
        ids = torch.as_tensor(table[r], device=DEV).long().clamp(min=0)
        mine = got[0][ids].transpose(1, 2).reshape(-1, hkv)[: n + steps].double()
        rows = (n + steps) * hq // hkv
        # (a sum of weights is off by what the weights are, 2^-18 of it, and by its own roundings)
        assert (mine.sum(0) - rows).abs().max() <= rows * 2.0 ** -17


def test_huge_logits_give_weights_of_at_most_one(zc):
    hq, hkv, page = 4, 2, 16
    for new in (1, 40):
        gen = torch.Generator(device=DEV).manual_seed(5)
        table, n_pages = ref.make_table(np.random.RandomState(5), [300], page)
        k, v = ref.make_pages(gen, n_pages, page, hkv, torch.bfloat16, False, DEV)
        q = (torch.randn(new, hq, D, generator=gen, device=DEV) * 2.0 ** 40).to(torch.bfloat16)
        scores = torch.zeros((n_pages, hkv, page), device=DEV)
        pool = zc.PagedKV(k, v, hq, max_req=1, max_rows=new, scored_rows=1)
        pool.attention_scored(q, i32(table), i32([0, new]), i32([300]), new, scores)
        settled(zc)
        assert torch.isfinite(scores).all() and scores.min() >= 0 and scores.max() <= new * hq // hkv


@pytest.mark.parametrize("new,bound", [([1, 3, 2], 2), ([40, 9, 130, 64], 64)])
def test_a_request_with_more_rows_than_the_bound(zc, new, bound):
    """What it does to its own scores is not said; the others' are as without it."""
    gen = torch.Generator(device=DEV).manual_seed(8)
    lengths = [n + 300 for n in new]
    table, n_pages = ref.make_table(np.random.RandomState(8), lengths, 16)
    k, v = ref.make_pages(gen, n_pages, 16, 2, torch.float16, False, DEV)
    q = torch.randn(sum(new), 8, D, generator=gen, device=DEV).half()
    row_start = [0] + np.cumsum(new).tolist()
    pool = zc.PagedKV(k, v, 8, max_req=len(new), max_rows=sum(new), scored_rows=4)
    got, want = (torch.zeros((n_pages, 2, 16), device=DEV) for _ in range(2))
    pool.attention_scored(q, i32(table), i32(row_start), i32(lengths), bound, got)
    pool.attention_scored(q, i32(table), i32(row_start), i32(lengths), max(new), want)
    settled(zc)
    assert torch.isfinite(got).all()
    for r, n in enumerate(new):
        if n <= bound:
            ids = torch.as_tensor(table[r], device=DEV).long()
            ids = ids[ids >= 0]
            # (the same weights, added up by another kernel where the bound decides which)
            assert (got[ids] - want[ids]).abs().max() <= 2.0 ** -16 * n * 4


def test_lengths_beyond_the_table(zc):
    gen = torch.Generator(device=DEV).manual_seed(9)
    table, n_pages = ref.make_table(np.random.RandomState(9), [112, 112], 16, 7)
    k, v = ref.make_pages(gen, n_pages, 16, 2, torch.float16, False, DEV)
    for new in (1, 40):
        q = torch.randn(2 * new, 8, D, generator=gen, device=DEV).half()
        pool = zc.PagedKV(k, v, 8, max_req=2, max_rows=2 * new, scored_rows=1)
        got, want = (torch.zeros((n_pages, 2, 16), device=DEV) for _ in range(2))
        pool.attention_scored(q, i32(table), i32([0, new, 2 * new]), i32([5000, 2 ** 31 - 1]), new, got)
        pool.attention_scored(q, i32(table), i32([0, new, 2 * new]), i32([112, 112]), new, want)
        settled(zc)
        assert torch.equal(got, want)


def test_a_captured_step_and_another_stream(zc):
    pool, args, _, before = scored_case(zc, "fp16", 8, 2, 16, [100, 900, 33], [1, 2, 1])
    q, table, row_start, kv, most = args
    kv2 = kv.clone()
    start = torch.nan_to_num(before, nan=0.0)
    scores, want = start.clone(), start.clone()
    pool.attention_scored(*args, want)
    out, lse = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty(q.shape[:2], device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    pool.attention_scored(q, table, row_start, kv2, most, scores, out=out, row_lse=lse, stream=side)
    side.synchronize()
    assert torch.equal(scores, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pool.attention_scored(q, table, row_start, kv2, most, scores, out=out, row_lse=lse)
    for lengths in ([101, 902, 34], [17, 300, 2]):
        kv2.copy_(i32(lengths))
        scores.copy_(start)
        want = start.clone()
        pool.attention_scored(q, table, row_start, i32(lengths), most, want)
        graph.replay()
        settled(zc)
        assert torch.equal(scores, want)
