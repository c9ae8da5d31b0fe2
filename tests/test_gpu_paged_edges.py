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
