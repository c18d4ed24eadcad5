"""Host side of user histories: devices, fault records, counts that no launch takes.  No device."""
import ctypes as C

import pytest
import torch

from test_history_refusals import PTR, cache, rows


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


class Library:
    """In the library's place: notes calls, and says that all is well."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or 0


class OnDevice:
    """A tensor of device `index`, as far as the binding looks at it."""
    dtype, device = torch.int64, "cuda"

    def __init__(self, index, words=4, contiguous=True):
        self.index, self.words, self.contiguous = index, words, contiguous

    def get_device(self):
        return self.index

    def numel(self):
        return self.words

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return PTR


@pytest.fixture
def device_0(b, monkeypatch):
    """The current device is 0, its current stream 7."""
    lib = Library()
    monkeypatch.setattr(b, "_lib", lib)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: {0: 7}[index], raising=False)
    monkeypatch.setattr(b, "_stream", lambda: 7)
    return lib


def test_a_record_is_checked_on_its_own_device(b, device_0):
    """Not on the current one's stream, which knows nothing of the record's calls."""
    assert b.rec_history_check(OnDevice(0)) == (b.REC_OK, -1, -1)
    assert device_0.calls == ["rec_history_check"]
    h = object.__new__(b.HistoryCache)
    h.fault = OnDevice(1)
    for call in (h.check, lambda: b.rec_history_check(OnDevice(1)), lambda: b.rec_history_check(OnDevice(-1))):
        with pytest.raises(ValueError):
            call()
    assert device_0.calls == ["rec_history_check"]


def test_records_that_a_kernel_would_write_past(b, device_0):
    """Four adjacent 64-bit words: fewer, others between them, or smaller ones are none."""
    small = OnDevice(0)
    small.dtype = torch.int32
    for fault in (OnDevice(0, words=3), OnDevice(0, contiguous=False), small):
        with pytest.raises(ValueError):
            b.rec_history_check(fault)
    assert device_0.calls == []


def test_pointers_that_no_load_of_their_type_takes(b):
    """32-bit and 64-bit words off their alignment: a scalar load rounds such an address down, an atomic faults."""
    from test_history_refusals import query, window
    h, odd = cache(b), cache(b, dev_fault=PTR + 4)
    raw = lambda name: getattr(b._lib, name)  # noqa: E731
    assert raw("rec_history_write")(C.byref(odd), C.byref(rows(b)), C.byref(rows(b)), b.REC_F32, PTR, 4, None) == b.REC_ERR_ARG
    assert raw("rec_history_read")(C.byref(odd), PTR, 4, b.REC_F32, PTR, PTR, None) == b.REC_ERR_ARG
    attend = lambda h, **kw: raw("rec_history_attend")(C.byref(h), C.byref(query(b, **kw)), None, 0, None)  # noqa: E731
    assert attend(odd) == b.REC_ERR_ARG
    for kw in (dict(dev_lengths=PTR + 2), dict(dev_pages_of=PTR + 1)):
        assert attend(h, **kw) == b.REC_ERR_ARG, kw
    for kw in (dict(dev_fault=PTR + 4), dict(dev_offsets=PTR + 2)):
        assert raw("rec_window_attend")(C.byref(window(b, **kw)), None) == b.REC_ERR_ARG, kw
    assert raw("rec_history_check")(PTR + 4, None, None, None) == b.REC_ERR_ARG


@pytest.mark.parametrize("kv_heads", [1, 2, 3, 1024])
def test_more_rows_than_a_launch_has_threads_for(b, kv_heads):
    """A wave has 16 rows of a head, a block four, and a launch under 2^32 threads: refused as such, before it fails."""
    h, r = cache(b, kv_heads=kv_heads), rows(b)
    blocks = lambda n: -(-(-(-n // 16) * kv_heads) // 4)  # noqa: E731
    first = next(n for n in range((1 << 30) // kv_heads - 200, (1 << 30) // kv_heads + 200) if blocks(n) * 256 >= 1 << 32)
    for n in (first, first + 1, 1 << 30):
        assert b._lib.rec_history_write(C.byref(h), C.byref(r), C.byref(r), b.REC_F32, PTR, n, None) == b.REC_ERR_OVERFLOW, n
        assert b._lib.rec_history_read(C.byref(h), PTR, n, b.REC_F32, PTR, PTR, None) == b.REC_ERR_OVERFLOW, n


@pytest.mark.parametrize("batch", [1 << 25, 1 << 26, (1 << 26) + 1, 1 << 27, (1 << 31) - 1])
def test_more_histories_than_a_launch_has_blocks_for(b, batch):
    """2^56 blocks of 256 threads are 2^64: refused as well, not as few as what is left of that in 64 bits."""
    from test_history_refusals import window
    w = window(b, batch=batch, tokens=1, heads=1 << 30, kv_heads=1 << 30)
    assert b._lib.rec_window_attend(C.byref(w), None) == b.REC_ERR_OVERFLOW


def test_tensors_that_require_grad_are_refused(b):
    """There is no backward pass, and a result without one would lose gradients without a word."""
    x = torch.zeros(10, 2, 64, dtype=torch.float16)
    y, at = x.clone().requires_grad_(), torch.zeros(10, dtype=torch.int64)
    h = object.__new__(b.HistoryCache)
    h._index, h.head_dim, h.kv_heads, h.device = 0, 64, 2, "cuda:0"
    calls = [lambda q, k, v: b.attend_window(q, k, v, at.int()), lambda q, k, v: h.write(k, v, at), lambda q, k, v: h.attend(q, at[:, None].int(), at.int())]
    for call, which in zip(calls, ((0, 1, 2), (1, 2), (0,))):
        for i in which:
            args = [y if j == i else x for j in range(3)]
            with pytest.raises(ValueError, match="backward"):
                call(*args)
            with torch.no_grad(), pytest.raises(ValueError) as e:      # what the call says next: not on a device
                call(*args)
            assert "backward" not in str(e.value)


@pytest.mark.parametrize("which", ["write", "attend", "window", "means", "select", "attend_selected", "attend_shared", "rotate"])
def test_tensors_with_a_tangent_are_refused(b, monkeypatch, which):
    """Forward-mode differentiation: a dual tensor does not require grad, and is one under torch.no_grad() too."""
    from torch.autograd import forward_ad
    monkeypatch.setattr(b, "_lib", None)

    class Here(torch.Tensor):
        def get_device(self):
            return 0

    on = lambda x: x.as_subclass(Here)  # noqa: E731
    h = object.__new__(b.HistoryCache)
    h._index, h.head_dim, h.kv_heads, h.device, h._means_shape, h._workspaces = 0, 64, 2, "cuda:0", (6, 2, 64), {}
    bf = dict(dtype=torch.bfloat16)
    q, out, means, k = (on(torch.zeros(s, **bf)) for s in ((3, 2, 4, 64), (3, 2, 4, 64), (6, 2, 64), (3, 2, 64)))
    table, n, chosen, prefix, one = (on(torch.zeros(s, dtype=torch.int32)) for s in ((3, 5), (3,), (3, 2, 2, 4), (7,), (1,)))
    w, f = on(torch.ones(64)), on(torch.zeros(32, dtype=torch.float64))
    call, args = dict(write=(lambda x, y: h.write(x, y, n.long()), (k, k)), attend=(lambda x, o: h.attend(x, table, n, out=o), (q, out)),
                      window=(lambda x, y, z: b.attend_window(x, y, z, n), (k, k, k)), means=(lambda m: h.summarise(n, m), (means,)),
                      select=(lambda x, m: h.select(x, m, table, n, 4, out=chosen), (q, means)),
                      attend_selected=(lambda x, o: h.attend_selected(x, chosen, table, n, out=o), (q, out)),
                      attend_shared=(lambda x, o: h.attend_shared(x, prefix, one, table, n, out=o), (q, out)),
                      rotate=(lambda x, y, e, v, z, o, p: b.rotate_heads(x, y, n, e, v, z, q_out=o, k_out=p), (k, k, f, w, w, k, k)))[which]
    with forward_ad.dual_level():
        for i, x in enumerate(args):
            dual = on(forward_ad.make_dual(x.as_subclass(torch.Tensor), torch.ones(x.shape, dtype=x.dtype)))
            assert forward_ad.unpack_dual(dual).tangent is not None and not dual.requires_grad
            with torch.no_grad(), pytest.raises(ValueError, match="derivative"):
                call(*args[:i], dual, *args[i + 1:])
        with pytest.raises(AttributeError):                     # no library: further than the checks
            call(*args)
    with pytest.raises(AttributeError):
        call(*args)
