"""The operators on full-precision pages, on the GPU, against plain references in 64 bits: block
tables, writes, reads, attention of single tokens and chunks with and without a window, the windowed
prompt, and all of them together up to prefill compression."""
import math

import numpy as np
import pytest
import torch

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


# ---------------------------------------------------------------- block tables and slot maps
def run_tables(zc, page, past, fresh, n_pages, next_, end, width, n_rows, seed=0):
    rng = np.random.RandomState(seed)
    ids = rng.permutation(n_pages).tolist()
    table = np.full((len(past), width), -7, dtype=np.int32)
    for r, p in enumerate(past):
        held = min(width, -(-max(0, p) // page))
        table[r, :held] = rng.randint(0, max(1, n_pages), held)
    want_table = table.tolist()
    want = ref.tables(page, past, fresh, ids, [next_, end], want_table, n_rows)
    step = zc.StepTables(len(past), n_rows)
    for t in (step.kv_len, step.row_start, step.slots, step.pos, step.free_state):
        t.fill_(-99)
    dev_table = i32(table)
    step.build(page, i32(past), i32(fresh), i32(ids), i32([next_, end, 0]), dev_table)
    torch.cuda.synchronize()
    got = [t.cpu().tolist() for t in (step.kv_len, step.row_start, step.slots, step.pos, step.free_state)]
    for name, g, w in zip(("kv_len", "row_start", "slots", "pos", "free_state"), got, want):
        assert g == w, name
    assert dev_table.cpu().tolist() == want_table


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("n_req", [1, 3, 64, 1023, 1024, 1025, 2500])
def test_tables_over_request_counts(zc, page, n_req):
    rng = np.random.RandomState(n_req)
    past, fresh = rng.randint(0, 600, n_req).tolist(), rng.randint(0, 40, n_req).tolist()
    width = -(-640 // page)
    run_tables(zc, page, past, fresh, n_pages=2 * n_req + 5, next_=1, end=2 * n_req + 5, width=width,
               n_rows=sum(fresh) + 11, seed=n_req)


@pytest.mark.parametrize("kw", [
    dict(past=[0], fresh=[0], n_pages=4, next_=0, end=4, width=2, n_rows=0),                         # nothing at all
    dict(past=[0], fresh=[1], n_pages=4, next_=3, end=4, width=1, n_rows=1),
    dict(past=[15, 16, 17], fresh=[1, 1, 1], n_pages=4, next_=0, end=4, width=2, n_rows=3),          # page borders
    dict(past=[0, 0, 0], fresh=[40, 40, 40], n_pages=9, next_=2, end=6, width=3, n_rows=120),        # the list runs out
    dict(past=[5, 5], fresh=[40, 40], n_pages=9, next_=0, end=99, width=3, n_rows=90),               # end beyond the list
    dict(past=[5, 5], fresh=[40, 40], n_pages=9, next_=7, end=4, width=3, n_rows=90),                # an empty list
    dict(past=[30, 0, 90], fresh=[40, 100, 3], n_pages=30, next_=0, end=30, width=4, n_rows=143),    # full table rows
    dict(past=[0, 3, 0], fresh=[0, 0, 0], n_pages=9, next_=0, end=9, width=3, n_rows=6),             # padding only
    dict(past=[-4, 10], fresh=[3, -2], n_pages=9, next_=0, end=9, width=3, n_rows=5),                # negative lengths
    dict(past=[7, 8], fresh=[50, 60], n_pages=30, next_=0, end=30, width=8, n_rows=70),              # fewer rows than tokens
])
def test_tables_edges(zc, kw):
    run_tables(zc, 16, **kw)


def test_tables_of_a_long_chunk(zc):
    run_tables(zc, 16, past=[100, 3, 0], fresh=[1, 300000, 17], n_pages=19000, next_=5, end=19000, width=18800,
               n_rows=300100)


# ---------------------------------------------------------------- writes and reads
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("page,heads,rows", [(16, 1, 1), (64, 8, 77), (128, 3, 130), (256, 32, 9)])
def test_write_places_rows_and_nothing_else(zc, dtype, heads_first, page, heads, rows):
    gen = torch.Generator(device=DEV).manual_seed(rows)
    n_pages = rows // page + 4
    k, v = ref.make_pages(gen, n_pages, page, heads, TYPES[dtype], heads_first, DEV)
    joint = torch.randn(rows, 3 * heads, D, generator=gen, device=DEV).to(TYPES[dtype])   # strided rows
    kr, vr = joint[:, heads:2 * heads], joint[:, 2 * heads:]
    slots = np.random.RandomState(rows).permutation(n_pages * page)[:rows]
    slots[::5] = [-1, n_pages * page, -2 ** 31, 2 ** 31 - 1][rows % 4]     # padding and slots beyond the pages
    want_k, want_v = k.clone(), v.clone()
    for i, s in enumerate(slots.tolist()):
        if 0 <= s < n_pages * page:
            want_k[s // page, s % page], want_v[s // page, s % page] = kr[i], vr[i]
    pool = zc.PagedKV(k, v, heads, max_req=1, max_rows=1)
    pool.write(kr, vr, i32(slots))
    torch.cuda.synchronize()
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    pool.write(kr[:0], vr[:0], i32(slots[:0]))     # no rows
    torch.cuda.synchronize()
    assert torch.equal(k, want_k)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("heads_first", [False, True])
@pytest.mark.parametrize("page,heads,l", [(16, 1, 1), (16, 8, 257), (64, 3, 64), (256, 2, 300)])
def test_read_gives_dense_rows(zc, dtype, heads_first, page, heads, l):
    gen = torch.Generator(device=DEV).manual_seed(l)
    table, n_pages = ref.make_table(np.random.RandomState(l), [l, l, l], page)
    k, v = ref.make_pages(gen, n_pages, page, heads, TYPES[dtype], heads_first, DEV)
    pool = zc.PagedKV(k, v, heads, max_req=1, max_rows=1)
    K, V = pool.read(i32(table), l)
    for r in range(3):
        a, b = ref.rows_of_request(k, v, table[r], l)
        assert torch.equal(K[r], a.transpose(0, 1)) and torch.equal(V[r], b.transpose(0, 1))
    # into a wider tensor, with a page that does not exist: zeros
    table[1, 0] = [-1, n_pages, 2 ** 31 - 1][l % 3]
    K2, V2 = (torch.full((3, heads, l + 3, D), 7.0, dtype=TYPES[dtype], device=DEV) for _ in range(2))
    pool.read(i32(table), l, K2[:, :, :l], V2[:, :, :l])
    torch.cuda.synchronize()
    n = min(page, l)
    assert (K2[1, :, :n] == 0).all() and (V2[1, :, :n] == 0).all() and torch.equal(K2[1, :, n:l], K[1, :, n:])
    assert torch.equal(K2[0, :, :l], K[0]) and torch.equal(V2[2, :, :l], V[2]) and (K2[:, :, l:] == 7).all()


# ---------------------------------------------------------------- attention over pages
def attention_case(zc, dtype, hq, hkv, page, past, new, window=0, sinks=0, heads_first=False, poison=True,
                   pad_rows=0, kv_len=None, strided=False, seed=0):
    """Compares one call with the 64-bit reference; returns its inputs for further use."""
    dt, rng = TYPES[dtype], np.random.RandomState(seed)
    gen = torch.Generator(device=DEV).manual_seed(seed + 1)
    kv = [p + n for p, n in zip(past, new)] if kv_len is None else list(kv_len)
    table, n_pages = ref.make_table(rng, kv, page)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, heads_first, DEV)
    clean_k, clean_v = k.clone(), v.clone()
    row_start = np.concatenate([[0], np.cumsum(new)])
    rows = int(row_start[-1]) + pad_rows
    if poison:
        # whatever no row may see holds NaN and infinities: the rest of a last page, spare pages, and pages that
        # have left the window, whose table entries are gone as well
        kept = torch.zeros(n_pages, page, dtype=torch.bool, device=DEV)
        for r, n in enumerate(kv):
            first = n - new[r]
            lo = max(0, first - window + 1) if window else 0
            for idx in range(-(-n // page)):
                t = torch.arange(idx * page, (idx + 1) * page, device=DEV)
                seen = (t < n) & ((t >= lo) | (t < sinks))
                kept[table[r, idx]] = seen
                if not seen.any():
                    table[r, idx] = [-1, n_pages + 5, -2 ** 31][idx % 3]
        for pool in (k, v):
            pool[~kept] = torch.tensor([math.nan, math.inf, -math.inf, math.nan], dtype=dt, device=DEV).repeat(D // 4)
    if strided:
        joint = torch.randn(rows, hq + 2 * hkv, D, generator=gen, device=DEV).to(dt)
        q = joint[:, :hq]
    else:
        q = torch.randn(rows, hq, D, generator=gen, device=DEV).to(dt)
    pool = zc.PagedKV(k, v, hq, max_req=len(kv), max_rows=rows)
    out = torch.full((rows, hq, D), 9.0, dtype=dt, device=DEV)
    lse = torch.full((rows, hq), 9.0, dtype=torch.float32, device=DEV)
    args = (q, i32(table), i32(row_start), i32(kv), max(max(new), 1))
    pool.attention(*args, window=window, sinks=sinks, out=out, row_lse=lse)
    settled(zc)
    vmax = clean_v.abs().max().double()
    for r, n in enumerate(kv):
        a, e = int(row_start[r]), int(row_start[r + 1])
        if a == e:
            continue
        ids = np.maximum(ref_table(table, n_pages)[r], 0)
        kr, vr = ref.rows_of_request(clean_k, clean_v, ids, n)
        for h in range(hq):
            o, l, mean_abs, largest, seen, total = ref.attend(q[a:e, h], kr[:, h // (hq // hkv)], vr[:, h // (hq // hkv)],
                                                              n - (e - a), window, sinks)
            t_out, t_lse = ref.tolerances(dt, o, mean_abs, largest, seen, total, vmax)
            some = seen > 0
            assert torch.isfinite(out[a:e, h]).all(), (r, h)
            bad = (out[a:e, h].double() - o).abs() - t_out
            assert bad[some].numel() == 0 or bad[some].max() <= 0, (r, h, bad.max().item(), t_out.max().item())
            assert (out[a:e, h][~some] == 0).all() and (lse[a:e, h][~some] == -math.inf).all()
            off = (lse[a:e, h].double() - l).abs()[some] - t_lse[some]
            assert off.numel() == 0 or off.max() <= 0, (r, h, off.max().item())
    end = int(row_start[-1])
    assert (out[end:] == 9).all() and (lse[end:] == 9).all()        # rows behind the last request
    return pool, args, out, lse


def ref_table(table, n_pages):
    """Table entries that name no page stand for pages that nothing reads."""
    return np.where((table < 0) | (table >= n_pages), 0, table)


DECODE = [
    dict(hq=1, hkv=1, page=16, past=[0], new=[1]),                                            # one key
    dict(hq=4, hkv=4, page=16, past=[15, 16, 17, 127, 128, 129], new=[1] * 6),
    dict(hq=32, hkv=8, page=64, past=[200, 511, 1, 0], new=[1] * 4, strided=True),
    dict(hq=8, hkv=1, page=128, past=[5000], new=[1]),                                        # one unit over all CTAs
    dict(hq=16, hkv=1, page=32, past=[777, 3], new=[1, 1]),                                   # 16 query heads a key head
    dict(hq=6, hkv=2, page=256, past=[1000, 256, 255], new=[1, 1, 1], heads_first=True),      # groups of 3
    dict(hq=14, hkv=2, page=16, past=[300, 40], new=[1, 1]),                                  # groups of 7
    dict(hq=32, hkv=32, page=64, past=[100, 900, 2048], new=[1] * 3),
    dict(hq=8, hkv=2, page=16, past=[60, 900, 3], new=[4, 3, 2]),                             # a few tokens each
    dict(hq=2, hkv=2, page=16, past=[70, 0, 200], new=[16, 9, 0]),                            # 16 rows, no rows
    dict(hq=4, hkv=2, page=64, past=[10, 20, 30], new=[1, 0, 1], pad_rows=5),
    dict(hq=4, hkv=1, page=16, past=[0] * 4, new=[1] * 4, kv_len=[0, 1, 0, 30]),              # rows that see nothing
    dict(hq=4, hkv=2, page=16, past=[0] * 3, new=[4, 3, 2], kv_len=[2, 0, 2]),
    dict(hq=8, hkv=2, page=16, past=[i * 7 % 390 for i in range(700)], new=[i % 2 for i in range(700)]),   # many requests
]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("kw", DECODE)
def test_single_tokens_and_few_rows(zc, dtype, kw):
    attention_case(zc, dtype, **kw)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 3), (16, 0), (33, 4), (100, 17), (128, 128), (500, 1), (4096, 4),
                                          (2 ** 31 - 1, 2 ** 31 - 1)])
def test_single_tokens_under_a_window(zc, dtype, window, sinks):
    attention_case(zc, dtype, 8, 2, 16, [0, 15, 90, 130, 640, 1500], [1, 1, 2, 1, 4, 1], window=window, sinks=sinks)
    attention_case(zc, dtype, 4, 4, 64, [33, 700, 2047], [1, 1, 1], window=window, sinks=sinks, heads_first=True)


CHUNK = [
    dict(hq=4, hkv=1, page=16, past=[0], new=[5]),
    dict(hq=1, hkv=1, page=16, past=[0, 3], new=[17, 300]),
    dict(hq=32, hkv=8, page=64, past=[0, 100, 700], new=[64, 1, 65], strided=True),
    dict(hq=8, hkv=2, page=128, past=[1000, 0, 5], new=[130, 0, 257], heads_first=True),
    dict(hq=6, hkv=2, page=32, past=[77, 300], new=[100, 43]),                                # groups of 3: 126 of 128 rows
    dict(hq=5, hkv=1, page=256, past=[500, 0], new=[60, 300]),
    dict(hq=16, hkv=1, page=16, past=[129, 31], new=[20, 8]),
    dict(hq=14, hkv=2, page=16, past=[129, 31], new=[40, 8], pad_rows=9),
    dict(hq=4, hkv=4, page=64, past=[6000], new=[33]),                                        # few rows over a long cache: in pieces
    dict(hq=8, hkv=1, page=16, past=[9000, 20], new=[100, 3]),
    dict(hq=8, hkv=8, page=16, past=[10, 0, 128, 127, 1], new=[256, 128, 127, 129, 40]),
    dict(hq=4, hkv=2, page=16, past=[0] * 4, new=[40, 30, 20, 33], kv_len=[13, 0, 20, 1]),    # rows before the first key
    dict(hq=8, hkv=2, page=16, past=[i * 3 % 90 for i in range(300)], new=[(i * 5) % 21 for i in range(300)]),
    dict(hq=2, hkv=1, page=16, past=[1] * 1500, new=[9 if i == 700 else 1 for i in range(1500)]),
]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("kw", CHUNK)
def test_chunks(zc, dtype, kw):
    attention_case(zc, dtype, **kw)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 5), (31, 0), (64, 4), (128, 128), (200, 130), (1000, 300), (4096, 4)])
def test_chunks_under_a_window(zc, dtype, window, sinks):
    attention_case(zc, dtype, 8, 2, 16, [0, 90, 1000, 130], [150, 33, 70, 1], window=window, sinks=sinks)
    attention_case(zc, dtype, 2, 2, 128, [700, 5000], [300, 140], window=window, sinks=sinks, heads_first=True)


def test_a_cache_whose_offsets_pass_32_bits(zc):
    """Pages over more than 4 GB per tensor; the requests' pages lie at both ends."""
    page, heads = 256, 8
    n_pages = 9000                                    # 9000 x 512 KB
    k, v = (torch.zeros(n_pages, page, heads, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    gen = torch.Generator(device=DEV).manual_seed(3)
    ids = [n_pages - 1, 0, n_pages - 2, 8500]
    for t in (k, v):
        t[ids] = torch.randn(4, page, heads, D, generator=gen, device=DEV).to(torch.bfloat16)
    n = 4 * page - 30
    kr, vr = ref.rows_of_request(k, v, np.array(ids), n)
    for new in (1, 40):
        q = torch.randn(new, heads, D, generator=gen, device=DEV).to(torch.bfloat16)
        pool = zc.PagedKV(k, v, heads, max_req=1, max_rows=new)
        out, lse = pool.attention(q, i32([ids]), i32([0, new]), i32([n]), new)
        settled(zc)
        for h in range(heads):
            o, l, mean_abs, largest, seen, total = ref.attend(q[:, h], kr[:, h], vr[:, h], n - new, 0, 0)
            t_out, t_lse = ref.tolerances(torch.bfloat16, o, mean_abs, largest, seen, total, vr.abs().max().double())
            assert ((out[:, h].double() - o).abs() <= t_out).all() and ((lse[:, h].double() - l).abs() <= t_lse).all()
    rows = torch.randn(2, heads, D, generator=gen, device=DEV).to(torch.bfloat16)
    pool.write(rows, rows, i32([n_pages * page - 1, 8800 * page]))
    K, V = pool.read(i32([[n_pages - 1], [8800]]), page)
    torch.cuda.synchronize()
    assert torch.equal(K[0, :, -1], rows[0]) and torch.equal(V[1, :, 0], rows[1])


@pytest.mark.parametrize("new", [[1, 1, 1], [2, 90, 40]])
def test_the_same_call_twice_gives_the_same_bits(zc, new):
    pool, args, out, lse = attention_case(zc, "bf16", 8, 2, 16, [3000, 900, 50], new)
    for _ in range(3):
        o2, l2 = pool.attention(*args)
        torch.cuda.synchronize()
        assert torch.equal(o2, out) and torch.equal(l2, lse)


@pytest.mark.parametrize("few", [True, False])
def test_a_captured_step_replays_with_other_lengths(zc, few):
    """Tables, write and attention captured once and replayed on new lengths of the same shapes."""
    dt, hq, hkv, page, n_req = torch.float16, 8, 2, 16, 3
    n_rows, max_new = (3, 1) if few else (200, 120)
    gen = torch.Generator(device=DEV).manual_seed(8)
    n_pages, width = 400, 100
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
    pool, step = zc.PagedKV(k, v, hq, max_req=n_req, max_rows=n_rows), zc.StepTables(n_req, n_rows)
    past, fresh, state = i32([0] * n_req), i32([1] * n_req), i32([0, n_pages, 0])
    table, free = i32(np.full((n_req, width), -1)), i32(np.random.RandomState(1).permutation(n_pages))
    q = torch.randn(n_rows, hq, D, generator=gen, device=DEV).to(dt)
    kr, vr = (torch.randn(n_rows, hkv, D, generator=gen, device=DEV).to(dt) for _ in range(2))
    out, lse = torch.empty(n_rows, hq, D, dtype=dt, device=DEV), torch.empty(n_rows, hq, device=DEV)

    def one_step():
        step.build(page, past, fresh, free, state, table)
        pool.write(kr, vr, step.slots)
        pool.attention(q, table, step.row_start, step.kv_len, max_new, out=out, row_lse=lse)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        one_step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            one_step()
    host_past = [0, 0, 0]
    plans = [[1, 1, 1], [1, 0, 1], [0, 1, 1]] if few else [[100, 1, 99], [0, 120, 3], [40, 40, 1]]
    state.copy_(i32([0, n_pages, 0]))
    table.fill_(-1)
    for new in plans * 2:
        past.copy_(i32(host_past))
        fresh.copy_(i32(new))
        q.normal_(generator=gen)
        kr.normal_(generator=gen)
        vr.normal_(generator=gen)
        torch.cuda.synchronize()
        graph.replay()
        settled(zc)
        state.copy_(step.free_state)
        host_past = [p + n for p, n in zip(host_past, new)]
        rs, tab = np.concatenate([[0], np.cumsum(new)]), table.cpu().numpy()
        assert step.kv_len.tolist() == host_past and step.free_state[2].item() == 0
        for r in range(n_req):
            a, e = rs[r], rs[r + 1]
            if a == e:
                continue
            kk, vv = ref.rows_of_request(k, v, tab[r], host_past[r])
            assert torch.equal(kk[-new[r]:], kr[a:e]) and torch.equal(vv[-new[r]:], vr[a:e])
            for h in range(hq):
                o, l, mean_abs, largest, seen, total = ref.attend(q[a:e, h], kk[:, h // 4], vv[:, h // 4],
                                                                  host_past[r] - new[r], 0, 0)
                t_out, t_lse = ref.tolerances(dt, o, mean_abs, largest, seen, total, v.abs().max().double())
                assert ((out[a:e, h].double() - o).abs() <= t_out).all()
                assert ((lse[a:e, h].double() - l).abs() <= t_lse).all()


@pytest.mark.parametrize("max_new", [1, 40])
def test_a_captured_step_forked_over_two_streams(zc, max_new):
    """Copies, a fill and the write on a second stream between the captured calls: what a call waits for may be a
    kernel, a copy or several of them."""
    pool, (q, table, row_start, kv_len, n), out, lse = attention_case(zc, "bf16", 8, 2, 16, [500, 20], [max_new] * 2)
    n_rows = q.shape[0]
    slots = i32(np.concatenate([np.asarray([int(table[r, p // 16]) * 16 + p % 16 for p in range(k - max_new, k)])
                                for r, k in enumerate(kv_len.tolist())]))
    rows = torch.randn(2, n_rows, 2, D, device=DEV).to(q.dtype)
    k_in, v_in, q_in = rows[0].clone(), rows[1].clone(), torch.zeros_like(q)
    got, got_lse = torch.empty_like(out), torch.empty_like(lse)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()

    def one_step():
        forked, joined = torch.cuda.Event(), torch.cuda.Event()
        k_in.zero_()
        forked.record(a)
        b.wait_event(forked)
        with torch.cuda.stream(b):
            k_in.copy_(rows[0])
            pool.write(k_in, v_in, slots)
            joined.record(b)
        got.fill_(7.0)
        q_in.copy_(q)
        a.wait_event(joined)
        pool.attention(q_in, table, row_start, kv_len, n, out=got, row_lse=got_lse)

    with torch.cuda.stream(a):
        one_step()
        a.synchronize()
        want, want_lse = got.clone(), got_lse.clone()
        pool.write(rows[0], rows[1], slots)
        first, first_lse = pool.attention(q, table, row_start, kv_len, n)
        a.synchronize()
        assert torch.equal(first, want) and torch.equal(first_lse, want_lse)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=a):
            one_step()
    for _ in range(5):
        pool.k_pages.view(-1, 2, D)[slots.long()] = 0
        got.zero_()
        q_in.zero_()
        settled(zc)
        graph.replay()
        settled(zc)
        assert torch.equal(got, want) and torch.equal(got_lse, want_lse)


def test_two_streams_with_workspaces_of_their_own(zc):
    a, args_a, out_a, lse_a = attention_case(zc, "fp16", 8, 2, 16, [4000, 100], [30, 60], seed=1)
    b, args_b, out_b, lse_b = attention_case(zc, "fp16", 8, 2, 16, [2000, 900, 1], [1, 1, 1], seed=2)
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(20):
        with torch.cuda.stream(sa):
            got.append((a.attention(*args_a), out_a, lse_a))
        with torch.cuda.stream(sb):
            got.append((b.attention(*args_b), out_b, lse_b))
    settled(zc)
    for (o, l), ow, lw in got:
        assert torch.equal(o, ow) and torch.equal(l, lw)


def test_wrong_tensors_are_refused(zc):
    pool, (q, table, row_start, kv_len, n), out, lse = attention_case(zc, "fp16", 8, 2, 16, [40], [3])
    bad = [dict(q=q.bfloat16()), dict(q=q[:, :4]), dict(table=table.long()), dict(table=table.T), dict(row_start=row_start[:1]),
           dict(kv_len=kv_len.float())]
    for b in bad:
        kw = {**dict(q=q, table=table, row_start=row_start, kv_len=kv_len), **b}
        with pytest.raises((zc.ZipCacheError, ValueError)):
            pool.attention(kw["q"], kw["table"], kw["row_start"], kw["kv_len"], n)
    with pytest.raises(zc.ZipCacheError, match="capacity"):
        big = torch.zeros(900000, 8, D, dtype=torch.float16, device=DEV)
        pool.attention(big, table, row_start, kv_len, 900000)
    with pytest.raises(zc.ZipCacheError):
        pool.write(q[:, :2].bfloat16(), q[:, :2].bfloat16(), i32([0, 1, 2]))
    with pytest.raises(zc.ZipCacheError):
        pool.write(q[:, :2], q[:, :2], i32([0, 1]))
    with pytest.raises(zc.ZipCacheError, match="capacity"):
        pool.read(table, table.shape[1] * 16 + 1)
    with pytest.raises(zc.ZipCacheError):
        zc.PagedKV(pool.k_pages, pool.v_pages.bfloat16(), 8)


def test_tensors_on_another_device_are_refused(zc):
    """Host tensors: the pointers would mean nothing to the kernels."""
    pool, (q, table, row_start, kv_len, n), out, lse = attention_case(zc, "fp16", 8, 2, 16, [40], [3])
    for i in range(4):
        args = [q, table, row_start, kv_len]
        args[i] = args[i].cpu()
        with pytest.raises(zc.ZipCacheError):
            pool.attention(*args, n)
    for kw in (dict(out=out.cpu()), dict(row_lse=lse.cpu())):
        with pytest.raises(zc.ZipCacheError):
            pool.attention(q, table, row_start, kv_len, n, **kw)
    rows, slots = q[:, :2].contiguous(), i32([0, 1, 2])
    for args in ((rows.cpu(), rows, slots), (rows, rows.cpu(), slots), (rows, rows, slots.cpu())):
        with pytest.raises(zc.ZipCacheError):
            pool.write(*args)
    dense = torch.empty(1, 2, 16, D, dtype=torch.float16)
    with pytest.raises(zc.ZipCacheError):
        pool.read(table, 16, dense, dense)
    with pytest.raises(zc.ZipCacheError):
        pool.read(table.cpu(), 16)
    with pytest.raises(zc.ZipCacheError):
        zc.PagedKV(pool.k_pages, pool.v_pages.cpu(), 8)
    with pytest.raises(zc.ZipCacheError):
        zc.PagedKV(pool.k_pages, pool.v_pages, 8, workspace=torch.zeros(pool.workspace_bytes, dtype=torch.uint8))
    step = zc.StepTables(1, 3)
    with pytest.raises(zc.ZipCacheError):
        step.build(16, kv_len.cpu(), kv_len, kv_len, i32([0, 1, 0]), table)
    cache = zc.ZipCache(torch.float16, 1, 8, 2, 16, 1, 0.4, device=DEV)
    x = torch.zeros(1, 8, 16, D, dtype=torch.float16, device=DEV)
    for args in ((x.cpu(), x[:, :2], x[:, :2]), (x, x[:, :2].cpu(), x[:, :2]), (x, x[:, :2], x[:, :2].cpu()),
                 (x.float(), x[:, :2], x[:, :2]), (x, x, x)):
        with pytest.raises(zc.ZipCacheError):
            cache.prefill_attention_window(*args, 4)
    settled(zc)


@pytest.mark.parametrize("max_new", [1, 70])
def test_steps_issued_without_a_pause(zc, max_new):
    """Tables, write and attention over the same buffers, step after step with nothing waited for: each kernel starts
    while the one before runs, and must see all that it wrote.  The same steps with a pause after every call give
    the bits to match."""
    dt, hq, hkv, page, n_req, steps = torch.bfloat16, 8, 2, 16, 5, 12
    n_pages, width = 600, 120
    rng = np.random.RandomState(max_new)
    plan = [i32(rng.randint(0, max_new + 1, n_req)) for _ in range(steps)]
    gen = torch.Generator(device=DEV).manual_seed(max_new)
    q = torch.randn(steps, n_req * max_new, hq, D, generator=gen, device=DEV).to(dt)
    kr, vr = (torch.randn(steps, n_req * max_new, hkv, D, generator=gen, device=DEV).to(dt) for _ in range(2))
    free = i32(rng.permutation(n_pages))

    def run(pause):
        k, v = (torch.zeros(n_pages, page, hkv, D, dtype=dt, device=DEV) for _ in range(2))
        pool = zc.PagedKV(k, v, hq, max_req=n_req, max_rows=n_req * max_new)
        turn = [zc.StepTables(n_req, n_req * max_new) for _ in range(2)]
        past, state, table = i32([0] * n_req), i32([0, n_pages, 0]), i32(np.full((n_req, width), -1))
        out, lse = torch.zeros_like(q), torch.zeros(steps, n_req * max_new, hq, device=DEV)
        settled(zc)
        for i in range(steps):
            step = turn[i & 1]
            for call in (lambda: step.build(page, past, plan[i], free, state, table),
                         lambda: pool.write(kr[i], vr[i], step.slots),
                         lambda: pool.attention(q[i], table, step.row_start, step.kv_len, max_new, out=out[i],
                                                row_lse=lse[i])):
                call()
                if pause:
                    torch.cuda.synchronize()
            past, state = step.kv_len, step.free_state
        settled(zc)
        return k, v, table, state, out, lse

    want = run(True)
    for _ in range(5):
        for g, w in zip(run(False), want):
            assert torch.equal(g, w)


def test_many_short_and_long_chunks(zc):
    """Items of one and of two tiles of rows in every order, through one place of Q after the other."""
    rng = np.random.RandomState(12)
    new = [int(n) for n in rng.choice([1, 2, 7, 31, 32, 33, 63, 64, 65, 100, 130], 48)]
    past = [int(p) for p in rng.randint(0, 700, 48)]
    attention_case(zc, "bf16", 8, 2, 16, past, new, seed=4)


# ---------------------------------------------------------------- a window over dense tensors
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("b,hq,hkv,l,window,sinks", [
    (1, 1, 1, 1, 1, 0), (2, 4, 4, 130, 1, 0), (1, 8, 2, 300, 64, 4), (2, 6, 2, 515, 100, 0), (1, 4, 2, 700, 128, 128),
    (1, 2, 1, 1000, 257, 300), (2, 8, 1, 257, 5000, 3), (1, 2, 2, 2100, 1024, 4), (1, 32, 8, 640, 500, 1)])
def test_windowed_prompt(zc, dtype, b, hq, hkv, l, window, sinks):
    dt = TYPES[dtype]
    gen = torch.Generator(device=DEV).manual_seed(l + window)
    # rows of a joint projection: [b, l, heads, D] seen as [b, heads, l, D]
    joint = torch.randn(b, l, hq + 2 * hkv, D, generator=gen, device=DEV).to(dt).transpose(1, 2)
    q, k, v = joint[:, :hq], joint[:, hq:hq + hkv], joint[:, hq + hkv:]
    cache = zc.ZipCache(dt, b, hq, hkv, l, 1, 0.4, device=DEV, guard_bytes=4096)
    out, lse = cache.prefill_attention_window(q, k, v, window, sinks)
    settled(zc)
    assert cache.check_guards()
    vmax = v.abs().max().double()
    for r in range(b):
        for h in range(hq):
            g = h // (hq // hkv)
            o, ls, mean_abs, largest, seen, total = ref.attend(q[r, h], k[r, g], v[r, g], 0, window, sinks)
            t_out, t_lse = ref.tolerances(dt, o, mean_abs, largest, seen, total, vmax)
            assert ((out[r, h].double() - o).abs() <= t_out).all(), (r, h)
            assert ((lse[r, h].double() - ls).abs() <= t_lse).all(), (r, h)


@pytest.mark.parametrize("window", [90, 5000])
def test_a_prompt_in_several_rounds_of_the_grid(zc, window):
    """352 items of different lengths: two full rounds of the CTAs and a part of one."""
    l, h = 2600, 32
    gen = torch.Generator(device=DEV).manual_seed(window)
    q, k, v = (torch.randn(1, h, l, D, generator=gen, device=DEV).half() for _ in range(3))
    cache = zc.ZipCache(torch.float16, 1, h, h, l, 1, 0.4, device=DEV)
    out, lse = cache.prefill_attention_window(q, k, v, window, 2)
    settled(zc)
    for i in range(h):
        o, ls, mean_abs, largest, seen, total = ref.attend(q[0, i], k[0, i], v[0, i], 0, window, 2)
        t_out, t_lse = ref.tolerances(torch.float16, o, mean_abs, largest, seen, total, v.abs().max().double())
        assert ((out[0, i].double() - o).abs() <= t_out).all(), i
        assert ((lse[0, i].double() - ls).abs() <= t_lse).all(), i


def test_a_window_of_the_whole_prompt_is_no_window(zc):
    """Within twice the tolerances' rounding terms of zc_prefill_attention, whose arithmetic is the same
    up to the order of its sums."""
    l = 600
    q, k, v = (torch.randn(1, h, l, D, device=DEV, generator=torch.Generator(device=DEV).manual_seed(h)).half()
               for h in (8, 2, 2))
    cache = zc.ZipCache(torch.float16, 1, 8, 2, l, 1, 0.4, device=DEV)
    o1, l1 = cache.prefill_attention(q, k, v)
    o2, l2 = cache.prefill_attention_window(q, k, v, l)
    settled(zc)
    for h in range(8):
        o, ls, mean_abs, largest, seen, total = ref.attend(q[0, h], k[0, h // 4], v[0, h // 4], 0, 0, 0)
        t_out, t_lse = ref.tolerances(torch.float16, o, mean_abs, largest, seen, total, v.abs().max().double())
        assert ((o1[0, h] - o2[0, h]).double().abs() <= 2 * t_out).all()
        assert ((l1[0, h] - l2[0, h]).double().abs() <= 2 * t_lse).all()


# ---------------------------------------------------------------- all together
@pytest.mark.parametrize("dtype,context,chunk", [("fp16", 512, 200), ("bf16", 777, 300)])
def test_a_prompt_through_pages_into_the_compressed_cache(zc, dtype, context, chunk):
    """A batch of prompts arrives in chunks: pages granted, rows written, chunk attention per step; the finished
    prompts are read back and compressed with the chunks' own row statistics; then a token is decoded from
    the compressed cache.  Every stage must be what the dense path gives: rows bit for bit, attention within
    its tolerance, salient sets and codes equal to the oracle's."""
    import zc_testlib as tl
    from workloads import make_decode_step, make_prefill
    w = tl.small_workload(context=context, batch=2, n_q_heads=8, n_kv_heads=2, dtype=dtype, outlier_fixed=0)
    Q, K, V = make_prefill(w, 0, DEV)
    page, b = 64, w.batch
    width = -(-context // page)
    n_pages = b * width
    kp, vp = (torch.zeros(n_pages, page, 2, D, dtype=w.torch_dtype, device=DEV) for _ in range(2))
    pool = zc.PagedKV(kp, vp, 8, max_req=b, max_rows=b * chunk)
    table = i32(np.full((b, width), -1))
    free, state = i32(np.random.RandomState(0).permutation(n_pages)), i32([0, n_pages, 0])
    O = torch.empty(b, 8, context, D, dtype=w.torch_dtype, device=DEV)
    lse = torch.empty(b, 8, context, device=DEV)
    done = 0
    while done < context:
        n = min(chunk, context - done)
        step = zc.StepTables(b, b * n)
        step.build(page, i32([done] * b), i32([n] * b), free, state, table)
        state = step.free_state.clone()
        rows = lambda t: t[:, :, done:done + n].transpose(1, 2).flatten(0, 1)  # noqa: E731  [b * n, heads, D]
        pool.write(rows(K), rows(V), step.slots)
        o, s = pool.attention(rows(Q), table, step.row_start, step.kv_len, n)
        O[:, :, done:done + n] = o.view(b, n, 8, D).transpose(1, 2)
        lse[:, :, done:done + n] = s.view(b, n, 8).transpose(1, 2)
        done += n
    assert state.tolist()[2] == 0
    Kd, Vd = pool.read(table, context)
    cache = tl.make_cache(w)
    probes = tl.probes_for(w)
    cache.prefill_compress_lse(Q, Kd, Vd, probes.tolist(), lse)
    settled(zc)
    assert torch.equal(Kd, K) and torch.equal(Vd, V)
    for r in range(b):
        for h in range(8):
            o, ls, mean_abs, largest, seen, total = ref.attend(Q[r, h], K[r, h // 4], V[r, h // 4], 0, 0, 0)
            t_out, t_lse = ref.tolerances(w.torch_dtype, o, mean_abs, largest, seen, total, V.abs().max().double())
            assert ((O[r, h].double() - o).abs() <= t_out).all() and ((lse[r, h].double() - ls).abs() <= t_lse).all()
    oc = tl.make_oracle(w)
    oc.prefill_compress(tl.to64(Q), tl.to64(K), tl.to64(V), probes)
    swaps, clean, _ = tl.compare_prefill_segment(w, cache, oc, oc.unit_ids)
    assert swaps == 0 and clean == len(oc.unit_ids)
    q, k, v = make_decode_step(w, 0, 0, DEV)
    cache.append(k, v)
    out = tl.to64(cache.decode_attention(q, False))
    oc.append(tl.to64(k), tl.to64(v))
    u = torch.finfo(w.torch_dtype).eps / 2
    for (bi, kv), o in oc.decode_attention(tl.to64(q), False).items():
        assert (np.abs(out[bi, kv * 4:(kv + 1) * 4] - o) <= 2e-3 + u * np.abs(o)).all()
    assert cache.check_guards()
