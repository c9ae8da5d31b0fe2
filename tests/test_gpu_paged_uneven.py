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
