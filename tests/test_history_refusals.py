"""What the calls of include/rec_history.h refuse, and shapes they accept: host code, no device."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


PTR = 0x10000      # aligned, never dereferenced: refused calls enqueue nothing


def cache(b, **kw):
    a = dict(dev_pages=PTR, num_pages=4, page_tokens=32, kv_heads=2, head_dim=64, format=b.REC_MX4, dev_fault=None)
    a.update(kw)
    return b.rec_history(*(a[f] for f, _ in b.rec_history._fields_))


def rows(b, dev=PTR, token_stride=128, head_stride=64):
    return b.rec_rows(dev, token_stride, head_stride)


def query(b, **kw):
    a = dict(dev_q=PTR, dev_out=PTR, batch_stride=256, query_stride=256, head_stride=64, dtype=b.REC_BF16, batch=3, queries=1,
             heads=4, dev_pages_of=PTR, table_stride=2, table_width=2, dev_lengths=PTR, scale=0.125, window=0, sinks=0, candidates=0)
    a.update(kw)
    return b.rec_query(*(a[f] for f, _ in b.rec_query._fields_))


def window(b, **kw):
    a = dict(q=rows(b), k=rows(b), v=rows(b), dev_out=PTR, dtype=b.REC_F16, batch=2, tokens=10, heads=2, kv_heads=2, head_dim=64,
             dev_offsets=PTR, scale=0.125, window=0, sinks=0, dev_fault=None)
    a.update(kw)
    return b.rec_window(*(a[f] for f, _ in b.rec_window._fields_))


@pytest.mark.parametrize("fmt,d,per_token", [("mx4", 32, 34), ("mx4", 64, 68), ("mx4", 128, 136), ("mx8", 32, 66), ("mx8", 64, 132), ("mx8", 128, 264)])
def test_bytes_of_a_cache(b, fmt, d, per_token):
    for page in (16, 32, 64, 128, 256):
        assert b.rec_history_bytes(cache(b, num_pages=5, page_tokens=page, kv_heads=3, head_dim=d, format=b._FORMATS[fmt])) == 5 * page * 3 * per_token


BAD_SHAPES = [dict(num_pages=0), dict(num_pages=-1), dict(num_pages=1 << 36), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512),
              dict(page_tokens=0), dict(page_tokens=-32), dict(kv_heads=0), dict(kv_heads=1025), dict(head_dim=96), dict(head_dim=0),
              dict(head_dim=256), dict(format=2), dict(format=-1)]


@pytest.mark.parametrize("bad", BAD_SHAPES, ids=str)
def test_shapes_that_no_cache_has(b, bad):
    h = cache(b, **bad)
    assert b.rec_history_bytes(h) == 0
    assert b.rec_history_write(h, rows(b), rows(b), b.REC_F32, None, 0) == b.REC_ERR_SHAPE
    assert b.rec_history_read(h, None, 0, b.REC_F32, None, None) == b.REC_ERR_SHAPE
    assert b.rec_history_attend_workspace_bytes(h, query(b)) == 0
    assert b.rec_history_attend(h, query(b)) == b.REC_ERR_SHAPE


def test_long_caches_are_counted_in_64_bits(b):
    assert b.rec_history_bytes(cache(b, num_pages=1 << 22, page_tokens=256, kv_heads=8, head_dim=128)) == (1 << 30) * 8 * 136


def _raw(b, name):
    return getattr(b._lib, name)


def test_write_refuses(b):
    f, h, slots = _raw(b, "rec_history_write"), cache(b), PTR
    call = lambda h=h, k=rows(b), v=rows(b), dt=b.REC_F32, s=slots, n=4: f(  # noqa: E731
        h and C.byref(h), k and C.byref(k), v and C.byref(v), dt, s, n, None)
    assert call(n=0, s=None) == b.REC_OK
    for kw in (dict(h=None), dict(k=None), dict(v=None), dict(dt=3), dict(dt=-1), dict(s=None), dict(s=PTR + 4), dict(n=-1),
               dict(h=cache(b, dev_pages=None)), dict(h=cache(b, dev_pages=PTR + 8)), dict(k=rows(b, dev=None)), dict(k=rows(b, dev=PTR + 8)),
               dict(v=rows(b, token_stride=130)), dict(v=rows(b, head_stride=66)), dict(dt=b.REC_F16, k=rows(b, token_stride=132)),
               dict(dt=b.REC_BF16, k=rows(b, head_stride=68))):
        assert call(**kw) == b.REC_ERR_ARG, kw
    assert call(n=1 << 31) == b.REC_ERR_OVERFLOW
    assert call(n=1 << 30) == b.REC_ERR_OVERFLOW        # times two heads


def test_read_refuses(b):
    f, h = _raw(b, "rec_history_read"), cache(b)
    call = lambda h=h, s=PTR, n=4, dt=b.REC_BF16, k=PTR, v=PTR: f(h and C.byref(h), s, n, dt, k, v, None)  # noqa: E731
    assert call(n=0, s=None, k=None, v=None) == b.REC_OK
    for kw in (dict(h=None), dict(s=None), dict(n=-1), dict(dt=9), dict(k=None), dict(v=None), dict(k=PTR + 2), dict(v=PTR + 8),
               dict(h=cache(b, dev_pages=None))):
        assert call(**kw) == b.REC_ERR_ARG, kw
    assert call(n=1 << 31) == b.REC_ERR_OVERFLOW


def test_attend_refuses(b):
    f = _raw(b, "rec_history_attend")
    call = lambda h=cache(b), q=query(b), ws=None, n=0: f(h and C.byref(h), q and C.byref(q), ws, n, None)  # noqa: E731
    assert call(q=query(b, batch=0)) == b.REC_OK
    assert call(q=query(b, queries=0)) == b.REC_OK
    for kw in (dict(dev_q=None), dict(dev_out=None), dict(dev_q=PTR + 8), dict(dev_out=PTR + 2), dict(dtype=b.REC_F32), dict(dtype=7),
               dict(batch=-1), dict(queries=-1), dict(heads=0), dict(heads=-2), dict(table_width=-1), dict(dev_pages_of=None),
               dict(dev_lengths=None), dict(window=-1), dict(sinks=-1), dict(candidates=2), dict(batch_stride=257),
               dict(query_stride=4), dict(head_stride=65)):
        assert call(q=query(b, **kw)) == b.REC_ERR_ARG, kw
    assert call(h=None) == b.REC_ERR_ARG and call(q=None) == b.REC_ERR_ARG
    assert call(h=cache(b, dev_pages=None)) == b.REC_ERR_ARG
    assert call(q=query(b, heads=3)) == b.REC_ERR_SHAPE
    assert call(q=query(b, table_width=1 << 26)) == b.REC_ERR_OVERFLOW
    assert call(q=query(b, queries=1 << 30)) == b.REC_ERR_OVERFLOW
    assert call(q=query(b, batch=1 << 30)) == b.REC_ERR_OVERFLOW


def test_attend_refuses_a_small_workspace(b):
    """One long history is divided among workgroups, so it needs one."""
    h, q = cache(b, num_pages=100000), query(b, batch=1, table_width=2000)
    need = b.rec_history_attend_workspace_bytes(h, q)
    f = _raw(b, "rec_history_attend")
    if need:
        assert f(C.byref(h), C.byref(q), None, need, None) == b.REC_ERR_ARG
        assert f(C.byref(h), C.byref(q), PTR, need - 1, None) == b.REC_ERR_ARG
        assert f(C.byref(h), C.byref(q), PTR + 8, need, None) == b.REC_ERR_ARG


def test_window_refuses(b):
    f = _raw(b, "rec_window_attend")
    assert f(None, None) == b.REC_ERR_ARG
    call = lambda **kw: f(C.byref(window(b, **kw)), None)  # noqa: E731
    assert call(tokens=0) == b.REC_OK and call(batch=0) == b.REC_OK
    for kw in (dict(q=rows(b, dev=None)), dict(k=rows(b, dev=PTR + 8)), dict(v=rows(b, token_stride=4)), dict(q=rows(b, head_stride=1)),
               dict(dev_out=None), dict(dev_out=PTR + 4), dict(dtype=b.REC_F32), dict(batch=-1), dict(tokens=-1), dict(heads=0),
               dict(kv_heads=0), dict(dev_offsets=None), dict(window=-5), dict(sinks=-1)):
        assert call(**kw) == b.REC_ERR_ARG, kw
    for kw in (dict(head_dim=48), dict(head_dim=256), dict(heads=3)):
        assert call(**kw) == b.REC_ERR_SHAPE, kw
    assert call(tokens=1 << 31) == b.REC_ERR_OVERFLOW
    assert call(tokens=1 << 30) == b.REC_ERR_OVERFLOW


def test_check_and_status(b):
    assert _raw(b, "rec_history_check")(None, None, None, None) == b.REC_ERR_ARG
    assert b.status_string(b.REC_ERR_VALUE) != b.status_string(99)


def test_python_refuses_what_the_library_cannot_see(b):
    with pytest.raises(ValueError):
        b.HistoryCache(4, 32, 2, 64, "mx6")
    with pytest.raises(b.RecError) as e:
        b.HistoryCache(4, 48, 2, 64)
    assert e.value.status == b.REC_ERR_SHAPE
    x = torch.zeros(10, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError):       # not on a device
        b.attend_window(x, x, x, torch.tensor([0, 10], dtype=torch.int32))
    with pytest.raises(ValueError):
        b.HistoryCache(4, 32, 2, 64, pages=torch.zeros(4 * 32 * 2 * 68, dtype=torch.uint8))
