"""Refusals of the operators that share pages and thin them out, which need no GPU: every call below is turned down by the
host-side checks, over addresses that are never dereferenced."""
import ctypes as C

import pytest
import torch

FAKE, ODD, HALF = C.c_void_p(0x200000), C.c_void_p(0x200002), C.c_void_p(0x200008)
EINVAL, ECAPACITY, EALIGN = -1, -2, -4


def at(i):
    """Addresses far apart."""
    return C.c_void_p(0x10000000 * (i + 1))


@pytest.fixture(scope="module")
def zc():
    from paper_2405_14256_b200 import build
    build.build()
    import paper_2405_14256_b200 as mod
    mod.load_library()
    return mod


def config(zc, **kw):
    base = dict(dtype=torch.bfloat16, n_q_heads=32, n_kv_heads=8, page_size=64, n_pages=100,
                strides=(64 * 8 * 128, 8 * 128, 128))
    base.update(kw)
    return zc.ZcPageConfig.make(**base)


@pytest.fixture
def pages(zc):
    h = C.c_void_p(0)
    assert zc.lib().zc_pages_init(FAKE, FAKE, C.byref(config(zc)), C.byref(h)) == 0
    yield h
    zc.lib().zc_pages_free(h)


STRIDES = (C.c_int64 * 2)(32 * 128, 128)
BIG = 1 << 40
SCORED = dict(q=at(0), strides=STRIDES, table=at(1), width=10, row_start=at(2), kv_len=at(3), n_req=4, n_rows=4, max_rows=1,
              window=0, sinks=0, first=at(4), scores=at(5), out=at(6), lse=at(7), ws=at(8), ws_bytes=BIG, logits=at(9),
              logits_bytes=BIG, stream=None)
SHARED = dict(q=at(0), strides=STRIDES, table=at(1), width=10, row_start=at(2), kv_len=at(3), n_req=4, n_rows=4, max_rows=1,
              starts=at(4), shared=at(10), n_groups=2, scores=at(5), out=at(6), lse=at(7), ws=at(8), ws_bytes=BIG,
              logits=at(9), logits_bytes=BIG, stream=None)
SELECT = dict(table=at(0), width=10, kv_len=at(1), n_req=4, scores=at(2), keep=at(3), recent=2, first=at(4), kept=at(5),
              max_keep=64, kept_len=at(6), stream=None)
COMPACT = dict(table=at(0), width=10, kv_len=at(1), n_req=4, kept=at(2), max_keep=64, kept_len=at(3), scores=at(4),
               free=at(5), n_free=50, state=at(6), out=at(7), stream=None)


@pytest.mark.parametrize("bad,code", [
    (dict(q=None), EINVAL), (dict(scores=None), EINVAL), (dict(lse=None), EINVAL), (dict(logits=None), EINVAL),
    (dict(out=None), EINVAL), (dict(ws=None), EINVAL), (dict(width=0), EINVAL), (dict(window=-1), EINVAL),
    (dict(sinks=-1), EINVAL), (dict(n_req=-1), EINVAL), (dict(max_rows=-1), EINVAL), (dict(width=1 << 25), EINVAL),
    (dict(scores=HALF), EALIGN), (dict(logits=HALF), EALIGN), (dict(first=ODD), EALIGN), (dict(q=HALF), EALIGN),
    (dict(ws_bytes=1000), ECAPACITY), (dict(logits_bytes=100 * 64 * 32 * 4 - 1), ECAPACITY),
    (dict(n_rows=13000 * 64, max_rows=64), ECAPACITY), (dict(strides=(C.c_int64 * 2)(32 * 128, 64)), EINVAL)])
def test_scored_attention_refuses(zc, pages, bad, code):
    assert zc.lib().zc_paged_attention_scored(pages, *{**SCORED, **bad}.values()) == code
    assert zc.lib().zc_paged_attention_scored(None, *SCORED.values()) == EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(starts=None), EINVAL), (dict(shared=None), EINVAL), (dict(n_groups=-1), EINVAL), (dict(max_rows=5, n_rows=20), EINVAL),
    (dict(logits=None), EINVAL), (dict(lse=None), EINVAL), (dict(starts=ODD), EALIGN), (dict(shared=ODD), EALIGN),
    (dict(scores=HALF), EALIGN), (dict(n_groups=1025), ECAPACITY), (dict(ws_bytes=43 << 20), ECAPACITY),
    (dict(logits_bytes=100), ECAPACITY), (dict(n_req=13001, n_rows=13001), ECAPACITY)])
def test_shared_attention_refuses(zc, pages, bad, code):
    assert zc.lib().zc_paged_attention_shared(pages, *{**SHARED, **bad}.values()) == code
    assert zc.lib().zc_paged_attention_shared(None, *SHARED.values()) == EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(table=None), EINVAL), (dict(kv_len=None), EINVAL), (dict(scores=None), EINVAL), (dict(keep=None), EINVAL),
    (dict(kept=None), EINVAL), (dict(kept_len=None), EINVAL), (dict(recent=-1), EINVAL), (dict(max_keep=-1), EINVAL),
    (dict(width=0), EINVAL), (dict(width=1 << 25), EINVAL), (dict(n_req=-1), EINVAL), (dict(n_req=1 << 29), EINVAL),
    (dict(table=ODD), EALIGN), (dict(kept=ODD), EALIGN), (dict(first=ODD), EALIGN), (dict(scores=ODD), EALIGN),
    (dict(kept=at(1)), EINVAL), (dict(kept_len=at(3)), EINVAL), (dict(kept=at(2)), EINVAL), (dict(kept_len=at(0)), EINVAL),
    (dict(kept_len=at(5)), EINVAL), (dict(kept_len=at(4)), EINVAL)])
def test_selection_refuses(zc, pages, bad, code):
    assert zc.lib().zc_page_select(pages, *{**SELECT, **bad}.values()) == code
    assert zc.lib().zc_page_select(None, *SELECT.values()) == EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(table=None), EINVAL), (dict(kv_len=None), EINVAL), (dict(kept=None), EINVAL), (dict(kept_len=None), EINVAL),
    (dict(free=None), EINVAL), (dict(state=None), EINVAL), (dict(out=None), EINVAL), (dict(max_keep=-1), EINVAL),
    (dict(n_free=-1), EINVAL), (dict(width=0), EINVAL), (dict(n_req=1 << 27), EINVAL), (dict(kept=ODD), EALIGN),
    (dict(scores=ODD), EALIGN), (dict(free=ODD), EALIGN), (dict(out=at(6)), EINVAL), (dict(free=at(0)), EINVAL),
    (dict(out=at(3)), EINVAL), (dict(scores=at(2)), EINVAL), (dict(out=at(5)), EINVAL), (dict(out=at(4)), EINVAL)])
def test_compaction_refuses(zc, pages, bad, code):
    assert zc.lib().zc_page_compact(pages, *{**COMPACT, **bad}.values()) == code
    assert zc.lib().zc_page_compact(None, *COMPACT.values()) == EINVAL


def test_calls_without_work_are_none(zc, pages):
    lib = zc.lib()
    assert lib.zc_paged_attention_scored(pages, *{**SCORED, "n_req": 0}.values()) == 0
    assert lib.zc_paged_attention_scored(pages, *{**SCORED, "n_rows": 0}.values()) == 0
    assert lib.zc_paged_attention_shared(pages, *{**SHARED, "max_rows": 0}.values()) == 0
    assert lib.zc_page_select(pages, *{**SELECT, "n_req": 0}.values()) == 0
    assert lib.zc_page_compact(pages, *{**COMPACT, "n_req": 0}.values()) == 0
    assert lib.zc_pages_launch_count(pages) == 0


def test_workspaces(zc):
    # 4 bytes per slot, query head and row; none where the chunk kernel is used
    assert zc.zc_scores_workspace(config(zc), 1) == 100 * 64 * 32 * 4
    assert zc.zc_scores_workspace(config(zc), 4) == 4 * 100 * 64 * 32 * 4
    assert zc.zc_scores_workspace(config(zc), 5) == zc.zc_scores_workspace(config(zc), 0) == 0
    small, large = (zc.zc_pages_shared_workspace(config(zc), 64, n) for n in (64, 128))
    assert large - small >= 64 * 32 * 2 * 132 * 4 and small > zc.zc_pages_workspace(config(zc), 64, 64)
    for call in (lambda: zc.zc_scores_workspace(config(zc), -1), lambda: zc.zc_pages_shared_workspace(config(zc), -1, 2),
                 lambda: zc.zc_scores_workspace(config(zc, page_size=48), 1)):
        with pytest.raises(zc.ZipCacheError, match="invalid argument"):
            call()
    with pytest.raises(zc.ZipCacheError, match="capacity"):
        zc.zc_pages_shared_workspace(config(zc), 13001, 2)
