"""Selection of the tokens to keep and compaction of pages, on the GPU: positions, lengths, rows and free lists against
plain Python, bit for bit."""
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


def make(zc, seed, page, hkv, lengths, dtype="fp16", heads_first=False, width=None):
    rng, gen = np.random.RandomState(seed), torch.Generator(device=DEV).manual_seed(seed)
    table, n_pages = ref.make_table(rng, lengths, page, width)
    k, v = ref.make_pages(gen, n_pages, page, hkv, TYPES[dtype], heads_first, DEV)
    scores = torch.rand((n_pages, hkv, page), generator=gen, device=DEV) ** 4
    pool = zc.PagedKV(k, v, hkv, max_req=0, max_rows=0)
    return pool, table, scores


def run_select(zc, pool, table, scores, lengths, keep, recent, first, max_keep):
    want, lens = er.select(scores, table.tolist(), pool.page_size, lengths, keep, recent,
                           first if first is not None else [0] * len(lengths), max_keep)
    kept, length = pool.select(i32(table), i32(lengths), scores, i32(keep), recent,
                               first=None if first is None else i32(first), max_keep=max_keep)
    settled(zc)
    assert length.tolist() == lens
    assert kept.tolist() == want
    return kept, length, want, lens


@pytest.mark.parametrize("page,hkv", [(16, 1), (64, 3), (256, 2)])
@pytest.mark.parametrize("n,keep,recent,first", [
    (1, 1, 0, 0), (1, 0, 0, 0), (2, 1, 0, 0), (2, 1, 1, 0), (33, 32, 0, 0), (500, 64, 32, 4), (511, 510, 0, 0), (512, 1, 0, 0),
    (2047, 300, 100, 16), (2049, 2000, 7, 0), (5000, 17, 5, 12), (9000, 4096, 1024, 0), (1000, 0, 0, 0), (1000, 50, 0, 50)])
def test_select_over_lengths(zc, page, hkv, n, keep, recent, first):
    lengths = [n, max(1, n // 2), n]
    pool, table, scores = make(zc, n + keep, page, hkv, lengths)
    run_select(zc, pool, table, scores, lengths, [keep, keep, max(0, keep - 1)], recent, [first, 0, first], max(1, keep))


def test_select_edges_of_the_rule(zc):
    """No tokens, negative numbers, budgets above max_keep, pinned and recent tokens that are more than the budget or than
    max_keep, pinned beyond the length, lengths beyond the table."""
    lengths = [0, -5, 100, 100, 100, 100, 100, 30, 5000]
    pool, table, scores = make(zc, 3, 16, 2, [max(0, min(n, 112)) for n in lengths], width=7)
    keep = [5, 5, -3, 90, 10, 10, 60, 64, 20]
    first = [0, 0, 2, 0, 30, 60, -4, 200, 3]
    run_select(zc, pool, table, scores, lengths, keep, 8, first, 40)
    run_select(zc, pool, table, scores, lengths, keep, 0, None, 40)


@pytest.mark.parametrize("n", [300, 1024, 7000])
def test_select_ties_and_odd_values(zc, n):
    """Equal scores keep the lower positions; signed zeros are equal; infinities, subnormals and negatives in order; NaN is
    the lowest."""
    pool, table, scores = make(zc, n, 16, 2, [n, n, n])
    odd = torch.tensor([0.0, -0.0, float("inf"), -float("inf"), float("nan"), 1e-42, -1e-42, 1.0, -1.0, 3e38], device=DEV)
    pick = torch.randint(0, odd.numel(), scores.shape, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    for keep in (n // 7, n // 2, n - 1):
        run_select(zc, pool, table, odd[pick], [n] * 3, [keep] * 3, 3, [0, 1, 2], keep)
        run_select(zc, pool, table, torch.zeros_like(scores), [n] * 3, [keep] * 3, 3, [0, 1, 2], keep)
    run_select(zc, pool, table, (scores * 4).floor(), [n] * 3, [n // 3] * 3, 0, None, n // 3)


def test_select_of_a_context_beyond_shared_memory(zc):
    """More candidates than are held: the rest is fetched again."""
    lengths = [70001, 49152, 49153]
    pool, table, scores = make(zc, 9, 256, 1, lengths)
    run_select(zc, pool, table, scores, lengths, [30000, 1000, 49152], 64, [4, 4, 0], 49152)
    run_select(zc, pool, table, (scores * 50).floor(), lengths, [30000, 1000, 49152], 0, None, 49152)


def test_select_with_a_page_that_is_none(zc):
    pool, table, scores = make(zc, 11, 16, 2, [100, 100])
    table[0, 2], table[1, 3] = -1, 10 ** 6
    run_select(zc, pool, table, scores, [100, 100], [60, 90], 4, [4, 0], 90)


def run_compact(zc, pool, table, scores, lengths, kept, lens, free=None, state=None, with_scores=True):
    max_keep = kept.shape[2]
    lists = kept.tolist()
    k2, v2, s2 = er.compact(pool.k_pages, pool.v_pages, scores, table.tolist(), pool.page_size, lengths, lists, lens, max_keep)
    if not with_scores:
        s2 = scores.clone()
    dev_free = None if free is None else i32(free)
    out = pool.compact(i32(table), i32(lengths), kept, i32(lens), scores=scores if with_scores else None,
                       free_pages=dev_free, free_state=None if free is None else i32(state))
    settled(zc)
    assert torch.equal(pool.k_pages, k2) and torch.equal(pool.v_pages, v2) and torch.equal(scores, s2)
    if free is not None:
        want_free, want_state = er.freed(table.tolist(), pool.page_size, lengths, lens, free, state, max_keep)
        assert dev_free.tolist() == want_free and out.tolist() == want_state


def random_kept(rng, lengths, lens, hkv, max_keep):
    kept = np.full((len(lengths), hkv, max_keep), -1, dtype=np.int32)
    for r, (n, m) in enumerate(zip(lengths, lens)):
        for h in range(hkv):
            if m <= max_keep:
                kept[r, h, :m] = np.sort(rng.permutation(max(n, m))[:m])
    return i32(kept)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("page,hkv,lengths,lens", [
    (16, 1, [1], [0]), (16, 1, [2, 2], [1, 2]), (16, 2, [300, 17, 0, 40], [128, 17, 0, 39]), (64, 8, [5000], [1000]),
    (64, 3, [700, 699, 64, 65], [640, 1, 63, 64]), (256, 2, [4000, 3999], [3990, 2048]), (32, 1, [20000], [9000]),
    (16, 32, [900] * 12, [450] * 12)])
def test_compact_moves_rows_and_pages(zc, dtype, heads_first, page, hkv, lengths, lens):
    """From one unit (clusters of eight) to hundreds (one CTA each), over and beyond a round's rows."""
    pool, table, scores = make(zc, sum(lengths), page, hkv, lengths, dtype, heads_first)
    rng = np.random.RandomState(len(lengths))
    kept = random_kept(rng, lengths, lens, hkv, max(1, max(lens)))
    room = sum(-(-n // page) for n in lengths)
    free = rng.randint(0, 1000, room + 5).tolist()
    run_compact(zc, pool, table, scores, lengths, kept, lens, free, [room + 2, room + 5, 7])


def test_compact_of_shapes_that_hurt_in_place(zc):
    """Everything shifts by one; the last rows move to the front; nothing moves; the first rows stay."""
    n, page, hkv = 3000, 64, 2
    for m, src in ((n - 1, np.arange(1, n)), (128, np.arange(n - 128, n)), (700, np.arange(700)),
                   (1500, np.concatenate([np.arange(10), np.arange(n - 1490, n)])), (1500, np.arange(0, n, 2))):
        pool, table, scores = make(zc, m, page, hkv, [n, n])
        kept = i32(np.broadcast_to(src, (2, hkv, m)).copy())
        run_compact(zc, pool, table, scores, [n, n], kept, [m, m], list(range(200)), [150, 200, 0])


def test_compact_without_lists_or_scores_and_the_free_list_s_edges(zc):
    lengths, lens = [200, 100, 90], [50, 100, 16]
    rng = np.random.RandomState(2)
    for free, state in ((None, None), ([1] * 40, [3, 40, 0]), ([1] * 40, [-2, 50, 0]), ([1] * 9, [99, 5, 0]), ([1] * 14, [14, 14, 1])):
        pool, table, scores = make(zc, 5, 16, 2, lengths)
        kept = random_kept(rng, lengths, lens, 2, 64)
        run_compact(zc, pool, table, scores, lengths, kept, lens, free, state, with_scores=free is not None)


def test_compact_leaves_requests_above_max_keep_alone(zc):
    lengths, lens = [300, 300, 300], [200, 64, 300]
    pool, table, scores = make(zc, 6, 16, 1, lengths)
    kept = random_kept(np.random.RandomState(1), lengths, lens, 1, 64)
    run_compact(zc, pool, table, scores, lengths, kept, lens, [0] * 40, [30, 40, 0])


def test_compact_past_32_bit_offsets(zc):
    """Pages whose strides put them beyond 2^32 bytes."""
    page, hkv, n = 16, 1, 64
    big = torch.zeros(5 << 30, dtype=torch.uint8, device=DEV).view(torch.float16)
    stride = (big.numel() // 6) // 8 * 8
    k = big.as_strided((6, page, hkv, D), (stride, D, D, 1))
    v = big[4096:].as_strided((6, page, hkv, D), (stride, D, D, 1))
    gen = torch.Generator(device=DEV).manual_seed(1)
    for t in (k, v):
        t.copy_(torch.randn(t.shape, generator=gen, device=DEV).half())
    scores = torch.rand((6, hkv, page), generator=gen, device=DEV)
    pool = zc.PagedKV(k, v, hkv, max_req=0, max_rows=0)
    table = np.array([[5, 0, 4, 2]], dtype=np.int32)
    kept = random_kept(np.random.RandomState(0), [n], [40], hkv, 40)
    run_compact(zc, pool, table, scores, [n], kept, [40], [9] * 4, [2, 4, 0])


def test_selection_and_compaction_captured_and_replayed_with_other_lengths(zc):
    page, hkv, cap = 16, 4, 640
    pool, table, scores = make(zc, 8, page, hkv, [cap, cap, cap])
    k0, v0, s0 = pool.k_pages.clone(), pool.v_pages.clone(), scores.clone()
    lengths, keep, dev_table = i32([600, 610, 620]), i32([512, 300, 100]), i32(table)
    free, state, out = i32([7] * 200), i32([150, 200, 0]), torch.zeros(3, dtype=torch.int32, device=DEV)
    kept, length = torch.empty((3, hkv, 512), dtype=torch.int32, device=DEV), torch.empty(3, dtype=torch.int32, device=DEV)

    def step():
        pool.select(dev_table, lengths, scores, keep, 32, kept=kept, kept_len=length)
        pool.compact(dev_table, lengths, kept, length, scores, free, state, out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for now, budget in (([640, 512, 513], [512, 512, 512]), ([16, 0, 333], [8, 8, 200])):
        for t, x in ((pool.k_pages, k0), (pool.v_pages, v0), (scores, s0)):
            t.copy_(x)
        lengths.copy_(i32(now))
        keep.copy_(i32(budget))
        free.fill_(7)
        graph.replay()
        settled(zc)
        want, lens = er.select(s0, table.tolist(), page, now, budget, 32, [0] * 3, 512)
        assert kept.tolist() == want and length.tolist() == lens
        k2, v2, s2 = er.compact(k0, v0, s0, table.tolist(), page, now, want, lens, 512)
        assert torch.equal(pool.k_pages, k2) and torch.equal(pool.v_pages, v2) and torch.equal(scores, s2)
        want_free, want_state = er.freed(table.tolist(), page, now, lens, [7] * 200, [150, 200], 512)
        assert free.tolist() == want_free and out.tolist() == want_state
