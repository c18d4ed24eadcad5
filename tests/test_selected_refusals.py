"""What the calls on chosen pages and on shared prefixes refuse: host code, no device."""
import ctypes as C

import pytest
import torch

from test_history_refusals import BAD_SHAPES, PTR, cache, query
from test_rotate_refusals import OnDevice, on


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


def ref(x):
    return x and C.byref(x)


def calls(b, h, q):
    """Every call with a query, all else in order, and its workspace's bytes."""
    lib = b._lib
    ws = 1 << 40
    return {
        "select": (lambda: lib.rec_history_select(ref(h), ref(q), PTR, 4, 1, 1, PTR, PTR, ws, None), lambda: lib.rec_history_select_workspace_bytes(ref(h), ref(q), 4)),
        "selected": (lambda: lib.rec_history_attend_selected(ref(h), ref(q), PTR, 4, PTR, ws, None), lambda: lib.rec_history_attend_selected_workspace_bytes(ref(h), ref(q), 4)),
        "shared": (lambda: lib.rec_history_attend_shared(ref(h), ref(q), PTR, 4, PTR, PTR, ws, None), lambda: lib.rec_history_attend_shared_workspace_bytes(ref(h), ref(q), 4)),
    }


@pytest.mark.parametrize("which", ["select", "selected", "shared"])
def test_queries(b, which):
    run = lambda h=cache(b), q=query(b): calls(b, h, q)[which]  # noqa: E731
    for bad in BAD_SHAPES:
        call, ask = run(h=cache(b, **bad))
        assert call() == b.REC_ERR_SHAPE and ask() == 0, bad
    for kw in (dict(batch=0), dict(queries=0)):
        call, ask = run(q=query(b, dev_q=None, dev_lengths=None, **kw))
        assert call() == b.REC_OK and ask() == 0
    for kw in (dict(dev_q=None), dict(dev_q=PTR + 8), dict(batch_stride=257), dict(query_stride=4), dict(head_stride=65), dict(dev_pages_of=None),
               dict(dev_pages_of=PTR + 2), dict(dev_lengths=None), dict(dev_lengths=PTR + 1)):
        assert run(q=query(b, **kw))[0]() == b.REC_ERR_ARG, kw
    for kw in (dict(dtype=b.REC_F32), dict(dtype=7), dict(batch=-1), dict(queries=-1), dict(heads=0), dict(table_width=-1), dict(window=-1), dict(window=5),
               dict(sinks=1), dict(candidates=2)):
        call, ask = run(q=query(b, **kw))
        assert call() == b.REC_ERR_ARG and ask() == 0, kw
    for h, q in ((None, query(b)), (cache(b), None)):
        call, ask = run(h, q)
        assert call() == b.REC_ERR_ARG and ask() == 0
    assert run(h=cache(b, dev_fault=PTR + 4))[0]() == b.REC_ERR_ARG
    assert run(q=query(b, heads=3))[0]() == b.REC_ERR_SHAPE
    for kw in (dict(table_width=1 << 26), dict(queries=1 << 30), dict(batch=1 << 30), dict(batch=1 << 25, queries=1, heads=2)):
        call, ask = run(q=query(b, **kw))
        assert call() == b.REC_ERR_OVERFLOW and ask() == 0, kw
    if which != "select":
        assert run(h=cache(b, dev_pages=None))[0]() == b.REC_ERR_ARG
        for out in (None, PTR + 2):
            assert run(q=query(b, dev_out=out))[0]() == b.REC_ERR_ARG


def test_choice(b):
    h, q = cache(b, num_pages=100000), query(b, table_width=9000)
    call = lambda means=PTR, count=4, first=1, last=1, out=PTR, ws=PTR, n=1 << 40: b._lib.rec_history_select(  # noqa: E731
        C.byref(h), C.byref(q), means, count, first, last, out, ws, n, None)
    for kw in (dict(means=None), dict(means=PTR + 8), dict(count=0), dict(count=-1), dict(first=-1), dict(last=0), dict(first=4), dict(first=2 ** 31 - 1, last=2 ** 31 - 1),
               dict(out=None), dict(out=PTR + 2), dict(ws=None), dict(ws=PTR + 8), dict(n=3 * 2 * 9000 * 8 - 1)):
        assert call(**kw) == b.REC_ERR_ARG, kw
    assert b.rec_history_select_workspace_bytes(h, q, 4) == 3 * 2 * 9000 * 8       # queries, kv heads, pages, a word each
    assert b.rec_history_select_workspace_bytes(h, q, 9000) == 0                   # all pages are chosen
    assert b.rec_history_select_workspace_bytes(h, query(b, table_width=512), 4) == 0       # a wave has a row's scores
    assert b.rec_history_select_workspace_bytes(h, query(b, table_width=513), 4) == 3 * 2 * 513 * 8
    assert b.rec_history_select_workspace_bytes(h, q, 0) == 0


@pytest.mark.parametrize("batch", [1, 8192, 1 << 20, 1 << 22, (1 << 22) + 9, 1 << 23, (1 << 23) + 5, 1 << 24, 1 << 30])
@pytest.mark.parametrize("width", [513, 5000, 1 << 20, (1 << 26) - 1, 1 << 26])
def test_choices_of_any_size_have_an_answer(b, batch, width):
    """Tiles of all rows may be 2^45 and more: what a wave has of them is a row's at most.  A wave or block chooses for a row of scores, 8 bytes a page."""
    h, q = cache(b, kv_heads=1, page_tokens=16, num_pages=100), query(b, batch=batch, queries=1, heads=1, table_width=width)
    call = b._lib.rec_history_select(C.byref(h), C.byref(q), PTR, 4, 1, 1, PTR, None, 0, None)
    need = b.rec_history_select_workspace_bytes(h, q, 4)
    threads = 64 * batch * (4 if width <= 2048 else 8 if width <= 4096 else 16)
    if threads < 1 << 32:
        assert need == 8 * batch * width and call == b.REC_ERR_ARG       # no workspace
    else:
        assert need == 0 and call == b.REC_ERR_OVERFLOW


@pytest.mark.parametrize("width", [2, 600, 9000])
def test_counts_that_a_block_steps_past(b, width):
    """A thread's next entry is up to 1024 behind its last: behind 2^31 - 1024 it does not fit 32 bits, and would be stored in front of the results."""
    h, q = cache(b), query(b, table_width=width)
    call = lambda count: b._lib.rec_history_select(C.byref(h), C.byref(q), None, count, 1, 1, PTR, PTR, 1 << 40, None)  # noqa: E731
    for count in (2 ** 31 - 1, 2 ** 31 - 64, 2 ** 31 - 1023):
        assert call(count) == b.REC_ERR_OVERFLOW and b.rec_history_select_workspace_bytes(h, q, count) == 0, count
    assert call(2 ** 31 - 1024) == b.REC_ERR_ARG       # no means
    assert max(range(1023, 2 ** 31 - 1024, 1024)) + 1024 < 2 ** 31


def test_chosen_pages(b):
    h, q = cache(b), query(b)
    call = lambda chosen=PTR, count=4: b._lib.rec_history_attend_selected(C.byref(h), C.byref(q), chosen, count, PTR, 1 << 40, None)  # noqa: E731
    for kw in (dict(chosen=None), dict(chosen=PTR + 2), dict(count=0), dict(count=-4)):
        assert call(**kw) == b.REC_ERR_ARG, kw
    assert call(count=1 << 26) == b.REC_ERR_OVERFLOW
    long = query(b, batch=1, table_width=4000)
    need = b.rec_history_attend_selected_workspace_bytes(h, long, 2000)
    assert need > 0                                                                # few pairs: parts
    for ws, n in ((None, need), (PTR, need - 1), (PTR + 8, need)):
        assert b._lib.rec_history_attend_selected(C.byref(h), C.byref(long), PTR, 2000, ws, n, None) == b.REC_ERR_ARG


def test_shared_prefixes(b):
    h, q = cache(b), query(b)
    call = lambda pages=PTR, width=5000, length=PTR, ws=PTR, n=1 << 40: b._lib.rec_history_attend_shared(  # noqa: E731
        C.byref(h), C.byref(q), pages, width, length, ws, n, None)
    for kw in (dict(pages=None), dict(pages=PTR + 2), dict(width=-1), dict(length=None), dict(length=PTR + 2), dict(ws=None), dict(ws=PTR + 8), dict(n=15)):
        assert call(**kw) == b.REC_ERR_ARG, kw
    assert call(width=1 << 26) == b.REC_ERR_OVERFLOW
    assert b.rec_history_attend_shared_workspace_bytes(h, q, 5000) > 0
    assert b.rec_history_attend_shared_workspace_bytes(h, q, 4) == 0       # little to read: one launch, without parts
    for kw in (dict(pages=None), dict(pages=PTR + 2), dict(length=None), dict(length=PTR + 2)):
        assert call(width=4, **kw) == b.REC_ERR_ARG, kw


@pytest.mark.parametrize("width", [1, 400, 4000, 40000])
@pytest.mark.parametrize("prefix", [1, 400, 4000, 40000])
def test_shared_prefixes_and_long_histories_come_in_64_parts_at_most(b, prefix, width):
    """What joins the parts of a row has room for 64; each takes the row's sums in 32 bits and two words more."""
    for per in (1, 64):
        q = query(b, batch=1, queries=1, heads=2 * per, table_width=width)
        parts, odd = divmod(b.rec_history_attend_shared_workspace_bytes(cache(b), q, prefix), 2 * per * (64 * 4 + 8))
        assert not odd and 0 <= parts <= 64 and (parts or prefix + width < 1000)


def test_means(b):
    call = lambda h=cache(b), which=PTR, n=3, means=PTR: b._lib.rec_history_summarise(ref(h), which, n, means, None)  # noqa: E731
    assert call(n=0, which=None, means=None) == b.REC_OK
    for kw in (dict(h=None), dict(which=None), dict(which=PTR + 2), dict(n=-1), dict(means=None), dict(means=PTR + 8), dict(h=cache(b, dev_pages=None)),
               dict(h=cache(b, dev_fault=PTR + 4))):
        assert call(**kw) == b.REC_ERR_ARG, kw
    for bad in BAD_SHAPES:
        assert call(h=cache(b, **bad)) == b.REC_ERR_SHAPE
    assert call(h=cache(b, kv_heads=1024), n=2 ** 31 - 1) == b.REC_ERR_OVERFLOW


def test_python_refuses_tensors_that_do_not_fit(b, monkeypatch):
    monkeypatch.setattr(b, "_lib", None)
    h = object.__new__(b.HistoryCache)
    h._index, h.head_dim, h.kv_heads, h.device, h._means_shape = 0, 64, 2, "cuda:0", (6, 2, 64)
    i32 = dict(dtype=torch.int32)
    q, means = on(torch.zeros(3, 2, 4, 64, dtype=torch.bfloat16)), on(torch.zeros(6, 2, 64, dtype=torch.bfloat16))
    table, n, chosen, prefix, one = (on(torch.zeros(s, **i32)) for s in ((3, 5), (3,), (3, 2, 2, 4), (7,), (1,)))
    good = dict(select=(q, means, table, n, 4), attend_selected=(q, chosen, table, n), attend_shared=(q, prefix, one, table, n))
    queries = [q.float(), q[..., :32], on(torch.zeros(3, 2, 4, 128, dtype=torch.bfloat16))[..., ::2], q[0, 0], torch.zeros_like(q.as_subclass(torch.Tensor)),
               on(torch.zeros(3, 2, 4, 64, dtype=torch.bfloat16, requires_grad=True))]
    tables = [table[:2], table.long(), table[0], on(torch.zeros(3, 10, **i32))[:, ::2]]
    lengths = [n[:2], n.long(), on(torch.zeros(6, **i32))[::2], n[:, None]]
    bad = {"select": {0: queries, 1: [means[:5], means.half(), means[:, :1], on(torch.zeros(6, 2, 128, dtype=torch.bfloat16))[..., ::2],
                                      on(torch.zeros(6, 2, 64, dtype=torch.bfloat16, requires_grad=True))], 2: tables, 3: lengths},
           "attend_selected": {0: queries, 1: [chosen.long(), chosen[:2], chosen[:, :1], chosen[:, :, :1], chosen[:, 0], on(torch.zeros(3, 2, 2, 8, **i32))[..., ::2]],
                               2: tables, 3: lengths},
           "attend_shared": {0: queries, 1: [prefix.long(), prefix[None], on(torch.zeros(14, **i32))[::2]], 2: [one.long(), n, prefix[:0]], 3: tables, 4: lengths}}
    monkeypatch.setattr(b.HistoryCache, "_result", lambda self, call, q, out: q)
    for name, places in bad.items():
        for place, values in places.items():
            for x in values:
                args = list(good[name])
                args[place] = x
                with pytest.raises(ValueError):
                    getattr(h, name)(*args)
    with pytest.raises(ValueError):
        h.select(*good["select"], out=chosen.long())
    for counts in (dict(count=0), dict(count=-1), dict(count=1 << 31), dict(count=(1 << 32) + 4), dict(first=-1), dict(first=5), dict(first=1 << 32),
                   dict(last=0), dict(last=5), dict(last=(1 << 32) + 1)):
        with pytest.raises(ValueError):
            h.select(*good["select"][:4], **{"count": 4, **counts})
    monkeypatch.undo()
    monkeypatch.setattr(b, "_lib", None)
    for name in ("attend_selected", "attend_shared"):
        for out in (q.half(), q[:2], on(torch.zeros(3, 2, 4, 128, dtype=torch.bfloat16))[..., ::2]):
            with pytest.raises(ValueError):
                getattr(h, name)(*good[name], out=out)
    for which, m in ((n.long(), means), (on(torch.zeros(6, **i32))[::2], means), (n, means[:5]), (n, means.float()), (table, means)):
        with pytest.raises(ValueError):
            h.summarise(which, m)
    assert isinstance(q, OnDevice)


@pytest.mark.parametrize("name", ["attend", "attend_selected", "attend_shared"])
def test_results_that_require_grad(b, monkeypatch, name):
    """What autograd knows of such a tensor would be of what it held before."""
    monkeypatch.setattr(b, "_lib", None)
    h = object.__new__(b.HistoryCache)
    h._index, h.head_dim, h.kv_heads, h.device, h._workspaces = 0, 64, 2, "cuda:0", {}
    q, out = (on(torch.zeros(3, 2, 4, 64, dtype=torch.bfloat16, requires_grad=r)) for r in (False, True))
    table, n, chosen, prefix, one = (on(torch.zeros(s, dtype=torch.int32)) for s in ((3, 5), (3,), (3, 2, 2, 4), (7,), (1,)))
    args = dict(attend=(q, table, n), attend_selected=(q, chosen, table, n), attend_shared=(q, prefix, one, table, n))[name]
    with pytest.raises(ValueError, match="backward"):
        getattr(h, name)(*args, out=out)
    with torch.no_grad(), pytest.raises(AttributeError):        # no library: further than the checks
        getattr(h, name)(*args, out=out)
