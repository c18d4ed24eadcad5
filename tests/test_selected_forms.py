"""The forms that choices of pages and attention behind shared prefixes take by their sizes.  No device."""
import ctypes as C

import pytest

from test_history_refusals import PTR, cache, query


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


def cached(b, kv, d, fmt="mx4", page=32):
    return cache(b, num_pages=100000, kv_heads=kv, head_dim=d, format=b._FORMATS[fmt], page_tokens=page)


def select(b, batch, queries, per, kv, d, width, count=16):
    h, q = cached(b, kv, d), query(b, batch=batch, queries=queries, heads=kv * per, table_width=width)
    st, *got = b.rec_probe_select_form(h, q, count)
    assert st == b.REC_OK
    need = b.rec_history_select_workspace_bytes(h, q, count)
    assert need == (8 * batch * queries * kv * width if got[0] == 2 else 0)
    return tuple(got)


def test_forms_of_a_choice(b):
    # one launch where a wave has a row's scores and a block's tiles do not take too long
    assert select(b, 1, 1, 2, 4, 64, 250) == (1, 2, 1)
    assert select(b, 16, 1, 4, 8, 128, 512) == (1, 4, 1)
    assert select(b, 256, 4, 4, 2, 64, 47) == (1, 16, 1)
    assert select(b, 64, 20, 2, 2, 32, 500) == (1, 16, 1)
    # two beyond that: 512 pages, and fewer where more than four rows are wide
    assert select(b, 16, 1, 4, 8, 128, 513) == (2, 4, 4)
    assert select(b, 16, 1, 8, 8, 128, 256) == (1, 8, 1) and select(b, 16, 1, 8, 8, 128, 257) == (2, 8, 4)
    assert select(b, 16, 3, 4, 8, 128, 300) == (2, 12, 4)
    assert select(b, 4, 1, 4, 2, 64, 2048)[2] == 4 and select(b, 4, 1, 4, 2, 64, 2049)[2] == 8 and select(b, 4, 1, 4, 2, 64, 4097)[2] == 16
    # more heads than a wave has rows; no scores where all pages are chosen
    assert select(b, 4, 3, 17, 2, 64, 600) == (2, 16, 4)
    assert select(b, 4, 3, 4, 2, 64, 600, 600)[0] == 1


def shared(b, batch, queries, per, kv, d, fmt, dtype, page, prefix, width):
    h, q = cached(b, kv, d, fmt, page), query(b, batch=batch, queries=queries, heads=kv * per, table_width=width, dtype=dtype)
    st, *got = b.rec_probe_shared_form(h, q, prefix)
    assert st == b.REC_OK
    parts = got[1] + (got[2] if got[2] > 1 else 0)
    assert b.rec_history_attend_shared_workspace_bytes(h, q, prefix) == parts * batch * queries * kv * per * (4 * d + 8)
    return tuple(got)


def test_forms_behind_a_prefix(b):
    bf, hf, joined, narrow, wide = b.REC_BF16, b.REC_F16, b.REC_SHARED_JOINED, b.REC_SHARED_NARROW, b.REC_SHARED_WIDE
    assert shared(b, 8, 1, 1, 4, 64, "mx8", hf, 32, 7, 1) == (joined, 0, 1)
    assert shared(b, 1, 1, 1, 1, 64, "mx4", bf, 32, 1000, 1000)[:2] == (joined, 0)
    assert shared(b, 1024, 1, 1, 2, 64, "mx4", bf, 32, 400, 1)[0] == narrow and shared(b, 1024, 1, 1, 2, 64, "mx4", bf, 32, 500, 1)[0] == wide
    assert shared(b, 64, 50, 4, 2, 32, "mx8", bf, 16, 63, 7) == (wide, 2, 1)
    assert shared(b, 256, 1, 4, 8, 128, "mx4", bf, 64, 128, 2)[0] == wide
    assert shared(b, 0, 1, 1, 2, 64, "mx4", bf, 32, 500, 1) == shared(b, 4, 0, 1, 2, 64, "mx4", bf, 32, 500, 1) == (joined, 0, 1)


@pytest.mark.parametrize("dtype", ["REC_BF16", "REC_F16"])
def test_parts_behind_a_prefix_are_all_at_work_at_once(b, dtype):
    """Four waves a history, head and part; a SIMD of 1024 holds three of the kernel behind a prefix, at 32 columns in mx8, else as many as without one."""
    for fmt, places in (("mx8", 3), ("mx4", 4)):
        for batch, own in ((64, 4000), (100, 1000), (150, 2000), (16, 8000)):
            form, _, parts = shared(b, batch, 1, 2, 4, 32, fmt, getattr(b, dtype), 32, 8000 // 32, own // 32)
            assert form == b.REC_SHARED_NARROW and parts == max(1, min(places * 1024 // (batch * 4 * 4), -(-own // 64) // 8)), (fmt, batch, parts)


def test_refused_calls_have_no_form(b):
    h = cache(b)
    for probe in (b.rec_probe_select_form, b.rec_probe_shared_form):
        assert probe(h, query(b, heads=3), 4)[0] == b.REC_ERR_SHAPE
        assert probe(cache(b, head_dim=48), query(b), 4)[0] == b.REC_ERR_SHAPE
        assert probe(h, query(b, window=5), 4)[0] == b.REC_ERR_ARG
        assert probe(h, query(b), -1)[0] == b.REC_ERR_ARG
        assert probe(h, query(b, table_width=1 << 26), 4)[0] == b.REC_ERR_OVERFLOW
    for probe in (b._lib.rec_probe_select_form, b._lib.rec_probe_shared_form):
        assert probe(C.byref(h), C.byref(query(b)), 4, None) == b.REC_ERR_ARG
