"""Full-precision pages, on the GPU: what one request's rows may depend on, logits that are not mild,
streams, and calls at the edge of what the documentation allows.  Values are compared with the 64-bit
references of zc_paged_ref under the tolerances derived there."""
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


def pool_of(zc, gen, dtype, hq, hkv, page, lengths, max_rows, seed=0, loud=1.0):
    """Pages of random rows for requests of these lengths: the handle and the table."""
    table, n_pages = ref.make_table(np.random.RandomState(seed), lengths, page)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dtype, False, DEV)
    k.mul_(loud)
    return zc.PagedKV(k, v, hq, max_req=len(lengths), max_rows=max_rows), i32(table)


# ---------------------------------------------------------------- whose rows decide
@pytest.mark.parametrize("hq,hkv", [(3, 1), (10, 2), (7, 1), (8, 2), (2, 2)])
def test_a_request_s_bits_do_not_depend_on_other_rows(zc, hq, hkv):
    """The second request's queries and the padding rows change, the first's do not, nor may its results: its tile
    of 128 rows holds some of theirs.  Logits of a standard deviation of about 6, so that a new maximum is due often."""
    dt, group = torch.bfloat16, hq // hkv
    new = [128 // group // 2 + 1, 128 // group + 3, 5]
    lengths = [2500, 1400, 40]
    rows = sum(new) + 40
    gen = torch.Generator(device=DEV).manual_seed(hq)
    pool, table = pool_of(zc, gen, dt, hq, hkv, 16, lengths, rows)
    q = (torch.randn(rows, hq, D, generator=gen, device=DEV) * 4).to(dt)
    args = (table, i32(np.concatenate([[0], np.cumsum(new)])), i32(lengths), max(new))
    out, lse = pool.attention(q, *args)
    settled(zc)
    assert torch.isfinite(out[:sum(new)]).all()
    for fill in (0.0, 40.0, math.nan, math.inf):
        for keep in range(3):
            other = torch.full_like(q, fill)
            a, e = sum(new[:keep]), sum(new[:keep + 1])
            other[a:e] = q[a:e]
            o, l = pool.attention(other, *args)
            settled(zc)
            assert torch.equal(o[a:e], out[a:e]) and torch.equal(l[a:e], lse[a:e]), (fill, keep)


@pytest.mark.parametrize("hq,hkv", [(3, 1), (10, 2), (7, 1)])
def test_the_same_bits_whatever_ran_before(zc, hq, hkv):
    """Groups of 3, 5 and 7 query heads leave rows of a tile that no copy writes: what other kernels left in the shared
    memory must not show."""
    dt, group = torch.bfloat16, hq // hkv
    new, lengths = [128 // group, 7 * (128 // group) + 5], [4000, 900]
    gen = torch.Generator(device=DEV).manual_seed(hq + 50)
    pool, table = pool_of(zc, gen, dt, hq, hkv, 16, lengths, sum(new))
    q = (torch.randn(sum(new), hq, D, generator=gen, device=DEV) * 4).to(dt)
    args = (q, table, i32([0, new[0], sum(new)]), i32(lengths), max(new))
    out, lse = pool.attention(*args)
    settled(zc)
    other, other_table = pool_of(zc, gen, dt, 4, 4, 64, [2000] * 8, 8 * 300)
    for fill in (1e4, math.nan, -3e38):
        loud = torch.full((8 * 300, 4, D), fill, dtype=dt, device=DEV)
        other.attention(loud, other_table, i32([300 * i for i in range(9)]), i32([2000] * 8), 300)
        o, l = pool.attention(*args)
        settled(zc)
        assert torch.equal(o, out) and torch.equal(l, lse), fill


# ---------------------------------------------------------------- streams
def busy(stream, ms=40):
    """Keeps a stream occupied for some time."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(int(ms * 1.9e6))


@pytest.mark.parametrize("own_stream", [False, True])
def test_the_first_call_on_another_stream_than_the_constructor_s(zc, own_stream):
    """The construction stream has long work in flight; a call at once on another stream, current or passed, must not
    meet counters that are not zero yet nor have its tables overwritten."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    new, lengths = [1, 1, 1], [4000, 3000, 50]
    k, v = ref.make_pages(gen, 450, 16, 2, torch.float16, False, DEV)
    q = torch.randn(3, 8, D, generator=gen, device=DEV).half()
    free, table = i32(np.random.RandomState(1).permutation(450)), i32(np.full((3, 250), -1))
    past, fresh, state = i32([n - 1 for n in lengths]), i32(new), i32([0, 450, 0])
    zeros = i32([0] * 3)
    first = zc.StepTables(3, sum(lengths))
    first.build(16, zeros, past, free, state, table)               # the cached tokens' pages
    state = first.free_state.clone()
    plain, step = zc.PagedKV(k, v, 8, max_req=3, max_rows=3), zc.StepTables(3, 3)
    step.build(16, past, fresh, free, state, table)
    out, lse = plain.attention(q, table, step.row_start, step.kv_len, 1)
    settled(zc)
    # memory of the workspace's and the tables' sizes holds something else than zeros when it is taken again
    junk = [torch.full((plain.workspace_bytes,), 0xFF, dtype=torch.uint8, device=DEV)] + [
        torch.full((n,), -1, dtype=torch.int32, device=DEV) for n in (3, 4, 3, 3, 3)]
    want = [t.clone() for t in (step.kv_len, step.row_start, step.slots, step.pos, step.free_state)]
    del plain, junk
    torch.cuda.synchronize()
    home, side = torch.cuda.Stream(), torch.cuda.Stream()
    busy(home)
    with torch.cuda.stream(home):
        pool, other = zc.PagedKV(k, v, 8, max_req=3, max_rows=3), zc.StepTables(3, 3)
        if own_stream:
            other.build(16, past, fresh, free, state, table, stream=side)
            o, l = pool.attention(q, table, other.row_start, other.kv_len, 1, stream=side)
    if not own_stream:
        with torch.cuda.stream(side):
            other.build(16, past, fresh, free, state, table)
            o, l = pool.attention(q, table, other.row_start, other.kv_len, 1)
    settled(zc)
    for got, w in zip((other.kv_len, other.row_start, other.slots, other.pos, other.free_state), want):
        assert torch.equal(got, w)
    assert torch.equal(o, out) and torch.equal(l, lse)


def test_allocated_outputs_belong_to_the_stream_that_writes_them(zc):
    """Memory that the current stream still uses, or will hand out again at once, is not what a call on another
    stream writes to."""
    gen = torch.Generator(device=DEV).manual_seed(6)
    pool, table = pool_of(zc, gen, torch.float16, 8, 2, 16, [900, 40], 8)
    q = torch.randn(4, 8, D, generator=gen, device=DEV).half()
    cache = zc.ZipCache(torch.float16, 1, 8, 2, 64, 1, 0.4, device=DEV)
    x = torch.randn(1, 12, 64, D, generator=gen, device=DEV).half()
    calls = {
        "attention": lambda **kw: pool.attention(q, table, i32([0, 2, 4]), i32([900, 40]), 2, **kw),
        "read": lambda **kw: pool.read(table, 40, **kw),
        "window": lambda **kw: cache.prefill_attention_window(x[:, :8], x[:, 8:10], x[:, 10:], 9, **kw),
        "prompt": lambda **kw: cache.prefill_attention(x[:, :8], x[:, 8:10], x[:, 10:], **kw),
    }
    side = torch.cuda.Stream()
    for name, call in calls.items():
        plain = [t.clone() for t in call()]
        torch.cuda.synchronize()
        held = [torch.empty_like(t) for t in plain]
        places = {t.data_ptr() for t in held}
        busy(torch.cuda.current_stream(), 20)
        for t in held:
            t.fill_(3.0)
        del held, t                       # free for the current stream, whose fill is still to come
        got = call(stream=side)
        assert not places & {t.data_ptr() for t in got}, name
        torch.cuda.synchronize()
        for g, w in zip(got, plain):
            assert torch.equal(g, w), name
        busy(side, 20)
        got = call(stream=side)
        places = {t.data_ptr() for t in got}
        del got, g                        # freed while the side stream has yet to write them
        held = [torch.empty_like(t) for t in plain]
        assert not places & {t.data_ptr() for t in held}, name
        torch.cuda.synchronize()
        del held
    settled(zc)


def test_a_dropped_handle_s_workspace_waits_for_the_streams_that_used_it(zc):
    gen = torch.Generator(device=DEV).manual_seed(7)
    pool, table = pool_of(zc, gen, torch.float16, 8, 2, 16, [900, 40], 8)
    q = torch.randn(4, 8, D, generator=gen, device=DEV).half()
    step = zc.StepTables(2, 4)
    args = (q, table, i32([0, 2, 4]), i32([900, 40]), 2)
    some = (i32([898, 38]), i32([2, 2]), i32([0]), i32([0, 0, 0]), table.clone())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy(side)
    pool.attention(*args, stream=side)
    step.build(16, *some, stream=side)
    size, at, slots = pool.workspace_bytes, pool.workspace.data_ptr(), step.slots.data_ptr()
    del pool, step
    again = [torch.empty(size, dtype=torch.uint8, device=DEV), torch.empty(4, dtype=torch.int32, device=DEV)]
    assert again[0].data_ptr() != at and again[1].data_ptr() != slots
    settled(zc)


def test_first_calls_of_several_threads_on_one_handle(zc):
    """The handle's tensor maps are made by whichever call comes first; each thread has a stream and a workspace."""
    from concurrent.futures import ThreadPoolExecutor
    from threading import Barrier
    gen = torch.Generator(device=DEV).manual_seed(9)
    n, gate, lib = 4, Barrier(4), zc.lib()
    table, n_pages = ref.make_table(np.random.RandomState(9), [300, 40], 16)
    k, v = ref.make_pages(gen, n_pages, 16, 2, torch.float16, False, DEV)
    table = i32(table)
    q = torch.randn(42, 8, D, generator=gen, device=DEV).half()
    steps = [(i32([0, 1, 2]), 1), (i32([0, 30, 42]), 30)]
    lengths = i32([300, 40])
    plain = zc.PagedKV(k, v, 8, max_req=2, max_rows=42)
    want = [plain.attention(q, table, rs, lengths, m) for rs, m in steps]
    streams = [torch.cuda.Stream() for _ in range(n)]
    works = [torch.zeros_like(plain.workspace) for _ in range(n)]
    settled(zc)

    def first(i, pool):
        rs, m = steps[i % 2]
        out, lse = torch.zeros_like(q), torch.zeros(42, 8, device=DEV)
        torch.cuda.synchronize()
        gate.wait()
        from paper_2405_14256_b200 import binding
        code = lib.zc_paged_attention(pool.handle, q.data_ptr(), binding._strides2(8 * D, D), table.data_ptr(), table.shape[1],
                                      rs.data_ptr(), lengths.data_ptr(), 2, 42, m, 0, 0, out.data_ptr(), lse.data_ptr(),
                                      works[i].data_ptr(), works[i].numel(), streams[i].cuda_stream)
        streams[i].synchronize()
        return code, out, lse

    with ThreadPoolExecutor(n) as threads:
        for _ in range(25):
            pool = zc.PagedKV(k, v, 8, max_req=2, max_rows=42, workspace=works[0])
            for i, (code, out, lse) in enumerate(threads.map(lambda i: first(i, pool), range(n))):
                rows = int(steps[i % 2][0][2])
                assert code == 0
                assert torch.equal(out[:rows], want[i % 2][0][:rows]) and torch.equal(lse[:rows], want[i % 2][1][:rows])
            assert zc.zc_pages_launch_count(pool.handle) == 2 * 1 + 2 * 2
    settled(zc)


# ---------------------------------------------------------------- logits that are not mild
@pytest.mark.parametrize("new", [1, 4, 60])
@pytest.mark.parametrize("dtype,power,sign", [("bf16", 55, -1), ("bf16", 59, -1), ("bf16", 55, 1), ("bf16", 16, -1),
                                              ("fp16", 14, -1), ("fp16", 14, 1), ("fp16", 11, 1)])
def test_rows_whose_logits_are_all_far_from_zero(zc, dtype, power, sign, new):
    """fp16 reaches logits of 2e9 and bf16 of 1e34.  Keys are so far apart then that nearly always a row's weight lies on
    its largest logit alone: the output is that value, and the log-sum-exp is that logit.
    From logits of 2^26 on the largest one's weight is 2^0 and the output exact.  Below, it is 2^x with x the rounding
    of the maximum, so that the weight is off by u, half a step of the type, against the sum (fp32: 2^-20 with the
    division), and the output is rounded once more: (1 + u)^2 (1 + 2^-20) - 1 of its size, 2^-25 where fp16 is not normal."""
    dt, lengths = TYPES[dtype], [1500, 700]
    u = torch.finfo(dt).eps / 2
    gen = torch.Generator(device=DEV).manual_seed(power + new)
    table, n_pages = ref.make_table(np.random.RandomState(power), lengths, 16)
    size = lambda *shape: torch.rand(shape, generator=gen, device=DEV) * 0.5 + 0.5  # noqa: E731
    k = (sign * size(n_pages, 16, 2, D) * 2.0 ** power).to(dt)
    v = torch.randn(n_pages, 16, 2, D, generator=gen, device=DEV).to(dt)
    q = (size(2 * new, 8, D) * 2.0 ** power).to(dt)
    pool = zc.PagedKV(k, v, 8, max_req=2, max_rows=2 * new)
    out, lse = pool.attention(q, i32(table), i32([0, new, 2 * new]), i32(lengths), new)
    settled(zc)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    checked = 0
    for r, n in enumerate(lengths):
        kk, vv = ref.rows_of_request(k, v, table[r], n)
        for h in range(8):
            logit = q[r * new:(r + 1) * new, h].double() @ kk[:, h // 4].double().T * (math.log2(math.e) / math.sqrt(D))
            assert (sign * logit).min() > 2.0 ** (2 * power) * 2
            hidden = torch.arange(n, device=DEV)[None] > torch.arange(n - new, n, device=DEV)[:, None]
            two, at = logit.masked_fill(hidden, -math.inf).topk(2, dim=1)
            # an fp32 logit is off by 136 * 2^-24 of its size (all terms have one sign): rows where the two largest
            # are further apart than twice that have one answer
            off = 136 * 2.0 ** -24 * two[:, 0].abs()
            sure = two[:, 0] - two[:, 1] > 2 * off + 64
            checked += int(sure.sum())
            rows = slice(r * new, (r + 1) * new)
            got, want = out[rows, h][sure].double(), vv[at[:, 0], h // 4][sure].double()
            far = two[sure, 0].abs()[:, None] > 2.0 ** 26 * (1 + 2.0 ** -10)
            slack = (2 * u + u * u + 2.0 ** -19) * want.abs() + 2.0 ** -25
            assert ((got - want).abs() <= torch.where(far, torch.zeros_like(slack), slack)).all()
            assert ((lse[rows, h].double() - two[:, 0]).abs() <= off + 2.0 ** -22 * two[:, 0].abs()).all()
    assert checked > 8 * new      # (of 16 * new rows)


def compare(zc, dt, q, k, v, table, row_start, lengths, max_rows, window=0, sinks=0):
    """One call against the 64-bit reference, every row."""
    hq, hkv = q.shape[1], k.shape[2]
    pool = zc.PagedKV(k, v, hq, max_req=len(lengths), max_rows=q.shape[0])
    out, lse = pool.attention(q, i32(table), i32(row_start), i32(lengths), max_rows, window=window, sinks=sinks)
    settled(zc)
    compare_rows(dt, out, lse, q, k, v, table, row_start, lengths, window, sinks)


def compare_rows(dt, out, lse, q, k, v, table, row_start, lengths, window=0, sinks=0, rows=None):
    hq, hkv = q.shape[1], k.shape[2]
    for r, n in enumerate(lengths):
        a, e = row_start[r], row_start[r + 1]
        some = e - a if rows is None else min(e - a, rows)
        if some == 0:
            continue
        kk, vv = ref.rows_of_request(k, v, table[r], n)
        for h in range(hq):
            o, l, mean_abs, largest, seen, total = ref.attend(q[a:a + some, h], kk[:, h // (hq // hkv)], vv[:, h // (hq // hkv)],
                                                              n - (e - a), window, sinks)
            t_out, t_lse = ref.tolerances(dt, o, mean_abs, largest, seen, total, vv.abs().max().double())
            off = (out[a:a + some, h].double() - o).abs() - t_out
            assert off.max() <= 0, (r, h, off.max().item())
            off = (lse[a:a + some, h].double() - l).abs() - t_lse
            assert off.max() <= 0, (r, h, off.max().item())


SHAPES = ["rising", "falling", "steps", "spike inside", "spike in the last block", "spike past 2^128", "two spikes", "wide"]


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("new,window,sinks", [([1, 1, 1], 0, 0), ([4, 1, 3], 700, 4), ([70, 200, 33], 0, 0), ([300, 20, 64], 900, 4)])
def test_maxima_that_are_renewed(zc, dtype, shape, new, window, sinks):
    """Logits that grow along the cache, or leap: every row's queries share a component c, and keys have multiples of it."""
    dt, hq, hkv, page = TYPES[dtype], 8, 2, 16
    lengths = [2300, 700, 330]
    gen = torch.Generator(device=DEV).manual_seed(len(shape) + sum(new))
    table, n_pages = ref.make_table(np.random.RandomState(3), lengths, page)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
    c = torch.randn(D, generator=gen, device=DEV)
    q = (torch.randn(sum(new), hq, D, generator=gen, device=DEV) * 0.5 + c).to(dt)
    # a key with m * c beside its noise has a logit of about 16 m (base 2)
    for r, n in enumerate(lengths):
        t = torch.arange(n, device=DEV)
        m = torch.zeros(n, device=DEV)
        if shape == "rising":
            m = 6.0 * t / n
        elif shape == "falling":
            m = 6.0 * (n - t) / n
        elif shape == "steps":
            m = (t // 64 % 7).float() * 0.5
        elif shape == "wide":
            m = torch.randn(n, generator=gen, device=DEV) * 1.5
        elif shape == "spike in the last block":
            m[n - 1 - new[r]] = 4.0
        elif shape == "spike past 2^128":
            m[n - n // 3] = 12.0
        else:
            m[n // 2 + 5] = 3.0
            if shape == "two spikes":
                m[n - n // 4] = 5.0
                m[3] = -9.0
        ids = torch.as_tensor(table[r], device=DEV).long()[t // page]
        k[ids, t % page] += (m[:, None] * c)[:, None].to(dt)
    compare(zc, dt, q, k, v, table, [0] + np.cumsum(new).tolist(), lengths, max(new), window, sinks)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("shape", ["rising", "spike", "spike past 2^128"])
@pytest.mark.parametrize("window,sinks", [(5000, 0), (700, 4)])
def test_maxima_that_are_renewed_in_a_windowed_prompt(zc, dtype, shape, window, sinks):
    dt, hq, hkv, l = TYPES[dtype], 4, 2, 1500
    gen = torch.Generator(device=DEV).manual_seed(len(shape))
    c = torch.randn(D, generator=gen, device=DEV)
    q = (torch.randn(1, hq, l, D, generator=gen, device=DEV) * 0.5 + c).to(dt)
    t = torch.arange(l, device=DEV)
    m = 6.0 * t / l if shape == "rising" else (t == 700) * (3.0 if shape == "spike" else 12.0)
    k = (torch.randn(1, hkv, l, D, generator=gen, device=DEV) + m[:, None] * c).to(dt)
    v = torch.randn(1, hkv, l, D, generator=gen, device=DEV).to(dt)
    cache = zc.ZipCache(dt, 1, hq, hkv, l, 1, 0.4, device=DEV)
    out, lse = cache.prefill_attention_window(q, k, v, window, sinks)
    settled(zc)
    for h in range(hq):
        o, ls, mean_abs, largest, seen, total = ref.attend(q[0, h], k[0, h // 2], v[0, h // 2], 0, window, sinks)
        t_out, t_lse = ref.tolerances(dt, o, mean_abs, largest, seen, total, v.abs().max().double())
        assert ((out[0, h].double() - o).abs() <= t_out).all(), h
        assert ((lse[0, h].double() - ls).abs() <= t_lse).all(), h


# ---------------------------------------------------------------- what the documentation allows
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("new,bound", [([1, 3, 2], 2), ([40, 9, 130, 64], 64), ([5, 300, 1], 33)])
def test_a_request_with_more_rows_than_the_bound(zc, dtype, new, bound):
    """The first `bound` rows of a request are right, the others may be left; nothing else is touched."""
    dt, hq, hkv = TYPES[dtype], 8, 2
    lengths = [n + 77 * (i + 1) for i, n in enumerate(new)]
    gen = torch.Generator(device=DEV).manual_seed(bound)
    table, n_pages = ref.make_table(np.random.RandomState(4), lengths, 16)
    k, v = ref.make_pages(gen, n_pages, 16, hkv, dt, False, DEV)
    rows = [0] + np.cumsum(new).tolist()
    q = torch.randn(rows[-1] + 7, hq, D, generator=gen, device=DEV).to(dt)
    out, lse = torch.full_like(q, 9.0), torch.full((rows[-1] + 7, hq), 9.0, device=DEV)
    pool = zc.PagedKV(k, v, hq, max_req=len(new), max_rows=rows[-1] + 7)
    pool.attention(q, i32(table), i32(rows), i32(lengths), bound, out=out, row_lse=lse)
    settled(zc)
    compare_rows(dt, out, lse, q, k, v, table, rows, lengths, rows=bound)
    for r, n in enumerate(new):
        left = slice(rows[r] + bound, rows[r + 1])
        if n > bound:
            right = pool.attention(q, i32(table), i32(rows), i32(lengths), max(new))
            same = (out[left] == 9).all(-1) | (out[left] == right[0][left]).all(-1)
            assert same.all()
    assert (out[rows[-1]:] == 9).all() and (lse[rows[-1]:] == 9).all()


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("hq,hkv,new,lengths", [(8, 2, [1, 1, 1], [900, 4000, 130]), (8, 1, [2, 1], [3000, 77]), (4, 4, [1, 1], [2000, 16])])
def test_single_tokens_are_off_by_the_output_s_rounding_alone(zc, dtype, hq, hkv, new, lengths):
    """A weight goes to the tensor cores as its value of the type and the rest of it, together off by u * u of it (u half
    a step; fp16: 2^-25 at least, where the rest is not normal).  So the output's bound has u of its own size and no u
    of the weighted values; the other terms are those of zc_paged_ref.tolerances."""
    dt = TYPES[dtype]
    u = torch.finfo(dt).eps / 2
    gen = torch.Generator(device=DEV).manual_seed(hq + len(new))
    table, n_pages = ref.make_table(np.random.RandomState(6), lengths, 16)
    k, v = ref.make_pages(gen, n_pages, 16, hkv, dt, False, DEV)
    v.abs_()                                     # outputs as large as the weighted values: nothing cancels
    rows = [0] + np.cumsum(new).tolist()
    q = torch.randn(rows[-1], hq, D, generator=gen, device=DEV).to(dt)
    pool = zc.PagedKV(k, v, hq, max_req=len(new), max_rows=rows[-1])
    out, lse = pool.attention(q, i32(table), i32(rows), i32(lengths), max(new))
    settled(zc)
    for r, n in enumerate(lengths):
        a, e = rows[r], rows[r + 1]
        kk, vv = ref.rows_of_request(k, v, table[r], n)
        for h in range(hq):
            o, l, mean_abs, largest, seen, total = ref.attend(q[a:e, h], kk[:, h // (hq // hkv)], vv[:, h // (hq // hkv)], n - (e - a), 0, 0)
            logit = 136 * 2.0 ** -24 * largest
            bound = (u * u + 2 * math.log(2) * logit + 2.0 ** -18)[:, None] * mean_abs + u * o.abs() + 2.0 ** -24
            if dt == torch.float16:
                bound = bound + (seen * 2.0 ** -25 * vv.abs().max().double() / total.clamp(min=1.0))[:, None]
            assert ((out[a:e, h].double() - o).abs() <= bound).all(), (r, h, ((out[a:e, h].double() - o).abs() / bound).max().item())


@pytest.mark.parametrize("page", [16, 256])
def test_a_page_id_that_no_pool_has_gives_no_slot(zc, page):
    """A page whose slots pass 2^31 - 1 cannot exist; its tokens have no slot instead of one of another page."""
    last = 2 ** 31 // page - 1                        # the largest page id that a pool can have
    ids = [last, last + 1, 2 ** 32 // page, 2 ** 31 - 1, 3]
    ids = [i for i in ids if i < 2 ** 31]
    n = len(ids) * page
    step, table = zc.StepTables(2, n + 1), i32([[5] + [-7] * len(ids), [last + 1, -7] + [-7] * (len(ids) - 1)])
    step.build(page, i32([page, page - 1]), i32([n, 1]), i32(ids), i32([0, len(ids), 0]), table)
    torch.cuda.synchronize()
    want = [i * page + t if i <= last else -1 for i in ids for t in range(page)] + [-1]
    assert step.slots.tolist() == want
    assert step.pos.tolist() == [page + i for i in range(n)] + [page - 1]
    assert table[0].tolist() == [5] + ids


def test_the_functions_beside_the_classes(zc):
    """zc_page_tables, zc_page_write, zc_page_read and zc_paged_attention take the tensors as they are, on a handle of
    zc_pages_init: what the classes give, bit for bit."""
    dt, hq, hkv, page = torch.bfloat16, 8, 2, 16
    gen = torch.Generator(device=DEV).manual_seed(11)
    past, new, n_pages, width = [100, 33], [3, 50], 40, 12
    rows = sum(new)
    k, v = ref.make_pages(gen, n_pages, page, hkv, dt, False, DEV)
    joint = torch.randn(rows, hq + 2 * hkv, D, generator=gen, device=DEV).to(dt)
    q, kr, vr = joint[:, :hq], joint[:, hq:hq + hkv], joint[:, hq + hkv:]
    held = np.full((2, width), -1, dtype=np.int32)
    held[0, :7], held[1, :3] = range(7), range(7, 10)
    free, state = i32(range(10, n_pages)), i32([0, n_pages - 10, 0])
    a_table, b_table = i32(held), i32(held)
    step = zc.StepTables(2, rows)
    step.build(page, i32(past), i32(new), free, state, a_table)
    pool = zc.PagedKV(k.clone(), v.clone(), hq, max_req=2, max_rows=rows)
    pool.write(kr, vr, step.slots)
    out, lse = pool.attention(q, a_table, step.row_start, step.kv_len, max(new), 40, 4)
    dense = pool.read(a_table, 80)

    cfg = zc.ZcPageConfig.make(dt, hq, hkv, page, n_pages, k.stride()[:3])
    work = torch.zeros(zc.zc_pages_workspace(cfg, 2, rows), dtype=torch.uint8, device=DEV)
    made = [torch.full((n,), -9, dtype=torch.int32, device=DEV) for n in (2, 3, rows, rows, 3)]
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    dense2 = [torch.empty_like(t) for t in dense]
    handle = zc.zc_pages_init(k, v, cfg)
    try:
        zc.zc_page_tables(page, i32(past), i32(new), free, state, b_table, *made)
        zc.zc_page_write(handle, kr, vr, made[2])
        zc.zc_paged_attention(handle, q, b_table, made[1], made[0], max(new), 40, 4, out2, lse2, work)
        zc.zc_page_read(handle, b_table, 80, *dense2)
        settled(zc)
        assert zc.zc_pages_launch_count(handle) == zc.zc_pages_launch_count(pool.handle) == 4
        with pytest.raises(zc.ZipCacheError, match="strides"):
            zc.zc_page_write(handle, kr, vr.contiguous(), made[2])
    finally:
        zc.zc_pages_free(handle)
    assert torch.equal(a_table, b_table) and torch.equal(out, out2) and torch.equal(lse, lse2)
    for a, b in zip((step.kv_len, step.row_start, step.slots, step.pos, step.free_state), made):
        assert torch.equal(a, b)
    assert torch.equal(pool.k_pages, k) and torch.equal(pool.v_pages, v)
    assert torch.equal(dense[0], dense2[0]) and torch.equal(dense[1], dense2[1])


@pytest.mark.parametrize("kw", [dict(max_rows=0), dict(max_req=0)])
def test_a_handle_that_only_copies_holds_no_workspace(zc, kw):
    table, n_pages = ref.make_table(np.random.RandomState(0), [30], 16)
    k, v = ref.make_pages(torch.Generator(device=DEV).manual_seed(1), n_pages, 16, 2, torch.float16, False, DEV)
    before = torch.cuda.memory_allocated()
    pool = zc.PagedKV(k, v, 4, **kw)
    assert torch.cuda.memory_allocated() == before and pool.workspace is None
    rows = torch.randn(2, 2, D, device=DEV).half()
    pool.write(rows, rows, i32([table[0, 0] * 16 + 3, table[0, 1] * 16]))
    K, V = pool.read(i32(table), 30)
    settled(zc)
    assert torch.equal(K[0, :, 3], rows[0]) and torch.equal(V[0, :, 16], rows[1])
    q = torch.zeros(1, 4, D, dtype=torch.float16, device=DEV)
    with pytest.raises(zc.ZipCacheError, match="workspace"):
        pool.attention(q, i32(table), i32([0, 1]), i32([30]), 1)
    shared = zc.PagedKV(k, v, 4, workspace=zc.PagedKV(k, v, 4).workspace, **kw)
    out, lse = shared.attention(q, i32(table), i32([0, 1]), i32([30]), 1)
    settled(zc)
    assert torch.isfinite(out).all()


def test_step_buffers_begin_as_zeros(zc):
    junk = torch.full((1 << 20,), -1, dtype=torch.int32, device=DEV)
    del junk
    home = torch.cuda.Stream()
    busy(home, 5)
    with torch.cuda.stream(home):
        step = zc.StepTables(3, 700)
    # (no stream of the reader's has been ordered behind the constructor's)
    with torch.cuda.stream(torch.cuda.Stream()):
        for t in (step.kv_len, step.row_start, step.slots, step.pos, step.free_state):
            assert (t == 0).all()


def test_a_shared_workspace_waits_for_the_streams_of_all_handles(zc):
    """Made by a handle on one stream, used by another handle on that one's own stream."""
    gen = torch.Generator(device=DEV).manual_seed(13)
    pool, table = pool_of(zc, gen, torch.float16, 8, 2, 16, [900, 40], 8)
    q = torch.randn(4, 8, D, generator=gen, device=DEV).half()
    args = (q, table, i32([0, 2, 4]), i32([900, 40]), 2)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = zc.PagedKV(pool.k_pages, pool.v_pages, 8, max_req=2, max_rows=8, workspace=pool.workspace)
    torch.cuda.synchronize()
    busy(side)
    with torch.cuda.stream(side):
        other.attention(*args)
    size, at = pool.workspace_bytes, pool.workspace.data_ptr()
    del pool, other
    again = torch.empty(size, dtype=torch.uint8, device=DEV)
    assert again.data_ptr() != at
    settled(zc)
