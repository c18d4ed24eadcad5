"""The form that a launch of cached attention takes by its size.  No device."""
import ctypes as C

import pytest

from test_history_refusals import PTR, cache, query


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


def form(b, batch, queries, heads, kv, d, fmt, dtype, page, width, window=0, sinks=0, candidates=0):
    h = cache(b, num_pages=100000, kv_heads=kv, head_dim=d, format=b._FORMATS[fmt], page_tokens=page)
    q = query(b, batch=batch, queries=queries, heads=heads, table_width=width, dtype=dtype, window=window, sinks=sinks, candidates=candidates)
    st, *got = b.rec_probe_history_form(h, q)
    assert st == b.REC_OK
    need = b.rec_history_attend_workspace_bytes(h, q)
    assert need == (got[1] * batch * queries * heads * (d * 4 + 8) if got[1] > 1 else 0)
    return tuple(got)


def test_forms(b):
    bf, hf = b.REC_BF16, b.REC_F16
    # one history of up to 200: four waves, no parts; up to 32768: parts of it, as many as work at once
    assert form(b, 1, 1, 4, 4, 64, "mx4", bf, 64, 4) == (4, 1, 1)
    assert form(b, 1, 1, 4, 4, 64, "mx4", bf, 64, 512) == (4, 64, 1)
    assert form(b, 32, 1, 32, 8, 128, "mx4", bf, 64, 512) == (4, 3, 1)
    assert form(b, 32, 1, 32, 8, 128, "mx4", bf, 64, 512, window=100, sinks=4) == (4, 1, 1)       # only four tiles of it are seen
    # many histories: two kv heads a wave, unless the rows of one fill more than half of it, or their number is odd
    assert form(b, 4096, 1, 4, 2, 32, "mx8", hf, 32, 7) == (1, 1, 2)
    assert form(b, 4096, 1, 4, 2, 128, "mx8", hf, 32, 7) == (1, 1, 1)
    assert form(b, 4096, 1, 18, 2, 32, "mx8", hf, 32, 7) == (1, 1, 1)
    assert form(b, 4096, 1, 3, 3, 32, "mx8", hf, 32, 7) == (1, 1, 1)
    # between: one wave a block and two parts; two waves; four where the longest may be long
    assert form(b, 1024, 1, 4, 2, 64, "mx4", bf, 64, 8) == (1, 2, 1)
    assert form(b, 512, 1, 4, 2, 64, "mx4", bf, 64, 8) == (2, 2, 1)
    assert form(b, 700, 1, 4, 2, 64, "mx8", hf, 64, 8) == (2, 1, 1)
    assert form(b, 1100, 1, 4, 2, 64, "mx4", bf, 32, 70) == (4, 1, 1)
    assert form(b, 1100, 1, 4, 2, 64, "mx4", bf, 32, 150) == (4, 2, 1)
    assert form(b, 5000, 1, 4, 2, 64, "mx4", bf, 32, 70) == (1, 1, 2)
    # candidates: rows of 16 by themselves
    assert form(b, 64, 50, 8, 4, 64, "mx4", bf, 32, 250, window=1000, sinks=4, candidates=1)[2] == 1
    # nothing to do, and no pages
    assert form(b, 0, 1, 4, 2, 64, "mx4", bf, 32, 70) == form(b, 5, 1, 4, 2, 64, "mx4", bf, 32, 0) == (1, 1, 1)


def test_a_divided_history_needs_its_workspace(b):
    h, q = cache(b, num_pages=100000), query(b, batch=1, table_width=2000)
    need = b.rec_history_attend_workspace_bytes(h, q)
    assert need > 0 and b.rec_probe_history_form(h, q)[2] > 1
    for ws, n in ((None, need), (PTR, need - 1), (PTR, 0), (PTR + 8, need)):
        assert b._lib.rec_history_attend(C.byref(h), C.byref(q), ws, n, None) == b.REC_ERR_ARG


def test_refused_queries_have_no_form(b):
    h = cache(b)
    assert b.rec_probe_history_form(h, query(b, heads=3))[0] == b.REC_ERR_SHAPE
    assert b.rec_probe_history_form(cache(b, head_dim=48), query(b))[0] == b.REC_ERR_SHAPE
    assert b.rec_probe_history_form(h, query(b, window=-1))[0] == b.REC_ERR_ARG
    assert b.rec_probe_history_form(h, query(b, table_width=1 << 26))[0] == b.REC_ERR_OVERFLOW
    assert b._lib.rec_probe_history_form(C.byref(h), C.byref(query(b)), None) == b.REC_ERR_ARG
