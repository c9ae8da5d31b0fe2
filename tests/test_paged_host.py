"""Refusals of the operators on full-precision pages that need no GPU: every call below is turned
down by the host-side checks, over addresses that are never dereferenced."""
import ctypes as C

import pytest
import torch

FAKE, ODD = C.c_void_p(0x20000), C.c_void_p(0x20008)
EINVAL, ECAPACITY, EALIGN = -1, -2, -4


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


@pytest.mark.parametrize("bad", [
    dict(dtype=7), dict(head_dim=64), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(n_pages=0),
    dict(n_pages=1 << 26, page_size=64), dict(n_q_heads=30), dict(n_kv_heads=0), dict(n_q_heads=8 * 17),
    dict(strides=(64 * 8 * 128, 8 * 128, 64)), dict(strides=(64 * 8 * 128, 8 * 128 + 4, 128)),
    dict(strides=(64 * 8 * 128, 0, 128)), dict(strides=(-64, 8 * 128, 128)), dict(strides=(1 << 40, 8 * 128, 128)),
])
def test_bad_page_configurations_are_refused(zc, bad):
    with pytest.raises(zc.ZipCacheError, match="invalid argument"):
        zc.zc_pages_workspace(config(zc, **bad), 8, 64)
    h = C.c_void_p(0)
    assert zc.lib().zc_pages_init(FAKE, FAKE, C.byref(config(zc, **bad)), C.byref(h)) == EINVAL and not h.value


def test_a_stride_of_an_extent_of_one_does_not_matter(zc):
    assert zc.zc_pages_workspace(config(zc, n_q_heads=4, n_kv_heads=1, strides=(64 * 128, 128, 0)), 8, 64) > 0
    assert zc.zc_pages_workspace(config(zc, n_pages=1, strides=(0, 8 * 128, 128)), 8, 64) > 0


def test_workspace_of_the_largest_calls(zc):
    # G = 4: 64 rows to an item
    assert zc.zc_pages_workspace(config(zc), 13000, 0) == zc.zc_pages_workspace(config(zc), 1, 12999 * 64) > 0
    for n_req, n_rows in [(13001, 0), (1, 13000 * 64), (13000, 64)]:
        with pytest.raises(zc.ZipCacheError, match="capacity"):
            zc.zc_pages_workspace(config(zc), n_req, n_rows)
    for n_req, n_rows in [(-1, 4), (4, -1)]:
        with pytest.raises(zc.ZipCacheError, match="invalid argument"):
            zc.zc_pages_workspace(config(zc), n_req, n_rows)


def test_init_refuses_null_and_misaligned_pages(zc):
    h, cfg = C.c_void_p(0), config(zc)
    f = zc.lib().zc_pages_init
    assert f(None, FAKE, C.byref(cfg), C.byref(h)) == EINVAL
    assert f(FAKE, None, C.byref(cfg), C.byref(h)) == EINVAL
    assert f(FAKE, ODD, C.byref(cfg), C.byref(h)) == EALIGN
    assert f(FAKE, FAKE, None, C.byref(h)) == EINVAL
    cfg.struct_size -= 4
    assert f(FAKE, FAKE, C.byref(cfg), C.byref(h)) == EINVAL
    zc.lib().zc_pages_free(None)
    assert zc.lib().zc_pages_launch_count(None) == 0


def test_tables_refusals(zc):
    f = zc.lib().zc_page_tables
    names = ["page_size", "n_req", "past", "fresh", "free_pages", "n_free", "free_state", "table", "width", "kv_len",
             "row_start", "n_rows", "slots", "pos", "free_out"]
    at = {n: C.c_void_p(0x10000 + 0x1000 * i) for i, n in enumerate(names)}
    good = {**at, **dict(page_size=16, n_req=4, n_free=8, width=4, n_rows=10)}
    for bad in [dict(page_size=0), dict(page_size=24), dict(n_req=0), dict(n_rows=-1), dict(n_free=-1), dict(width=0),
                dict(width=1 << 27)] + [
            {n: None} for n in names if n not in ("page_size", "n_req", "n_free", "width", "n_rows")]:
        kw = {**good, **bad}
        assert f(*[kw[n] for n in names], None) == EINVAL, bad
    inputs, outputs = ("past", "fresh", "free_pages", "free_state"), ("table", "kv_len", "row_start", "slots", "pos", "free_out")
    for i in inputs:
        for o in outputs:
            for shift in (-8, 0, 8):   # outputs that begin, or end, inside an input
                kw = {**good, o: C.c_void_p(at[i].value + shift)}
                assert f(*[kw[n] for n in names], None) == EINVAL, (i, o, shift)
    for n in inputs + outputs:
        kw = {**good, n: C.c_void_p(at[n].value + 2)}
        assert f(*[kw[n] for n in names], None) == EALIGN, n


def test_write_and_read_refusals(zc, pages):
    lib = zc.lib()
    rs, bad_rs = (C.c_int64 * 2)(1024, 128), (C.c_int64 * 2)(1024, 132)
    assert lib.zc_page_write(None, FAKE, FAKE, rs, FAKE, 3, None) == EINVAL
    assert lib.zc_page_write(pages, FAKE, FAKE, rs, FAKE, -1, None) == EINVAL
    assert lib.zc_page_write(pages, None, FAKE, rs, FAKE, 3, None) == EINVAL
    assert lib.zc_page_write(pages, FAKE, FAKE, rs, None, 3, None) == EINVAL
    assert lib.zc_page_write(pages, FAKE, FAKE, bad_rs, FAKE, 3, None) == EINVAL
    assert lib.zc_page_write(pages, FAKE, FAKE, None, FAKE, 3, None) == EINVAL
    assert lib.zc_page_write(pages, FAKE, ODD, rs, FAKE, 3, None) == EALIGN
    assert lib.zc_page_write(pages, FAKE, FAKE, rs, C.c_void_p(0x20002), 3, None) == EALIGN
    assert lib.zc_page_write(pages, None, None, rs, None, 0, None) == 0          # nothing to do
    ks, bad_ks = (C.c_int64 * 3)(8 * 640 * 128, 640 * 128, 128), (C.c_int64 * 3)(8, 4, 128)
    assert lib.zc_page_read(pages, FAKE, 10, 2, 641, FAKE, FAKE, ks, None) == ECAPACITY
    assert lib.zc_page_read(pages, FAKE, 10, 2, 0, FAKE, FAKE, ks, None) == EINVAL
    assert lib.zc_page_read(pages, FAKE, 10, 0, 64, FAKE, FAKE, ks, None) == EINVAL
    assert lib.zc_page_read(pages, None, 10, 2, 64, FAKE, FAKE, ks, None) == EINVAL
    assert lib.zc_page_read(pages, FAKE, 10, 2, 64, FAKE, FAKE, bad_ks, None) == EINVAL
    assert lib.zc_page_read(pages, FAKE, 10, 2, 64, ODD, FAKE, ks, None) == EALIGN
    assert lib.zc_page_read(pages, C.c_void_p(0x20002), 10, 2, 64, FAKE, FAKE, ks, None) == EALIGN
    assert lib.zc_page_read(None, FAKE, 10, 2, 64, FAKE, FAKE, ks, None) == EINVAL
    assert lib.zc_pages_launch_count(pages) == 0


def test_attention_refusals(zc, pages):
    f = zc.lib().zc_paged_attention
    names = ["p", "q", "qs", "table", "width", "row_start", "kv_len", "n_req", "n_rows", "max_rows", "window", "sinks", "out",
             "lse", "ws", "ws_bytes"]
    strides = (C.c_int64 * 2)(32 * 128, 128)
    ws = zc.zc_pages_workspace(config(zc), 4, 40)
    good = dict(p=pages, q=FAKE, qs=strides, table=FAKE, width=10, row_start=FAKE, kv_len=FAKE, n_req=4, n_rows=40,
                max_rows=10, window=0, sinks=0, out=FAKE, lse=FAKE, ws=FAKE, ws_bytes=ws)
    call = lambda **kw: f(*[{**good, **kw}[n] for n in names], None)  # noqa: E731
    for n in ("p", "q", "qs", "table", "row_start", "kv_len", "out", "ws"):
        assert call(**{n: None}) == EINVAL, n
    for bad in [dict(n_req=-1), dict(n_rows=-1), dict(max_rows=-1), dict(window=-1), dict(sinks=-1), dict(width=0),
                dict(width=1 << 25), dict(qs=(C.c_int64 * 2)(32 * 128, 132)), dict(qs=(C.c_int64 * 2)(32 * 128, 0)),
                dict(qs=(C.c_int64 * 2)(64, 128)), dict(qs=(C.c_int64 * 2)(-4096, 128))]:
        assert call(**bad) == EINVAL, bad
    for n in ("q", "out", "ws"):
        assert call(**{n: ODD}) == EALIGN, n
    for n in ("lse", "table", "row_start", "kv_len"):
        assert call(**{n: C.c_void_p(0x20002)}) == EALIGN, n
    assert call(ws_bytes=1024) == ECAPACITY and call(ws_bytes=1024, max_rows=1) == ECAPACITY
    # nothing to do
    assert call(n_req=0) == 0 and call(n_rows=0) == 0 and call(max_rows=0) == 0


def test_windowed_prompt_refusals(zc):
    cfg = zc.ZcConfig.make(torch.float16, 1, 4, 4, 64, 8, 0.5)
    nbytes, _ = zc.zc_cache_bytes(cfg)
    lib, h = zc.lib(), C.c_void_p(0)
    assert lib.zc_cache_init(C.c_void_p(0x10000), nbytes, C.byref(cfg), C.byref(h)) == 0
    try:
        ks = (C.c_int64 * 3)(4 * 64 * 128, 64 * 128, 128)
        odd = (C.c_int64 * 3)(4 * 64 * 128, 64 * 128, 132)
        f = lib.zc_prefill_attention_window
        assert f(h, FAKE, FAKE, FAKE, 64, ks, ks, 0, 0, FAKE, FAKE, None) == EINVAL
        assert f(h, FAKE, FAKE, FAKE, 64, ks, ks, -3, 0, FAKE, FAKE, None) == EINVAL
        assert f(h, FAKE, FAKE, FAKE, 64, ks, ks, 4, -1, FAKE, FAKE, None) == EINVAL
        assert f(h, FAKE, FAKE, FAKE, 0, ks, ks, 4, 0, FAKE, FAKE, None) == EINVAL
        assert f(h, FAKE, FAKE, FAKE, 65, ks, ks, 4, 0, FAKE, FAKE, None) == ECAPACITY
        assert f(h, FAKE, FAKE, FAKE, 64, odd, ks, 4, 0, FAKE, FAKE, None) == EINVAL
        assert f(h, FAKE, FAKE, FAKE, 64, ks, ks, 4, 0, FAKE, None, None) == EINVAL
        assert f(h, FAKE, ODD, FAKE, 64, ks, ks, 4, 0, FAKE, FAKE, None) == EALIGN
        assert f(None, FAKE, FAKE, FAKE, 64, ks, ks, 4, 0, FAKE, FAKE, None) == EINVAL
    finally:
        lib.zc_cache_free(h)
