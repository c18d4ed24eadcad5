"""What rec_rotate_heads() and rotate_heads() refuse: host code, no device."""
import ctypes as C

import pytest
import torch

PTR = 0x10000      # aligned, never dereferenced: refused calls enqueue nothing


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


def turn(b, **kw):
    rows = lambda **r: b.rec_rows(r.get("dev", PTR), r.get("token_stride", 256), r.get("head_stride", 64))  # noqa: E731
    a = dict(q=rows(), k=rows(), q_out=rows(), k_out=rows(), dtype=b.REC_BF16, heads=4, kv_heads=2, head_dim=64, tokens=10,
             dev_positions=PTR, wide=0, pairs=32, dev_frequencies=PTR, interleaved=0, eps=1e-6, dev_q_weight=PTR, dev_k_weight=PTR)
    a.update({k: rows(**v) if k in ("q", "k", "q_out", "k_out") else v for k, v in kw.items()})
    return b.rec_turn(*(a[f] for f, _ in b.rec_turn._fields_))


def call(b, **kw):
    return b._lib.rec_rotate_heads(C.byref(turn(b, **kw)), None)


def test_nothing_to_do(b):
    assert call(b, tokens=0, q=dict(dev=None)) == b.REC_OK
    assert call(b, heads=0, kv_heads=0, q=dict(dev=None), k=dict(dev=None)) == b.REC_OK


def test_arguments(b):
    assert b._lib.rec_rotate_heads(None, None) == b.REC_ERR_ARG
    for what in ("q", "k", "q_out", "k_out"):
        for bad in (dict(dev=None), dict(dev=PTR + 8), dict(token_stride=257), dict(head_stride=65)):
            assert call(b, **{what: bad}) == b.REC_ERR_ARG, (what, bad)
    for kw in (dict(dtype=3), dict(dtype=-1), dict(tokens=-1), dict(heads=-1), dict(kv_heads=-1), dict(wide=2), dict(interleaved=2),
               dict(eps=-1e-6), dict(eps=float("nan")), dict(dev_positions=None), dict(dev_positions=PTR + 2), dict(wide=1, dev_positions=PTR + 4),
               dict(dev_frequencies=None), dict(dev_frequencies=PTR + 4), dict(dev_q_weight=PTR + 4), dict(dev_k_weight=PTR + 8)):
        assert call(b, **kw) == b.REC_ERR_ARG, kw
    for kw in (dict(head_dim=48), dict(head_dim=256), dict(head_dim=0), dict(pairs=4), dict(pairs=40), dict(pairs=-8), dict(pairs=64)):
        assert call(b, **kw) == b.REC_ERR_SHAPE, kw


def test_rows_that_overlap(b):
    """Two results in one place: whichever was stored last."""
    for bad in (dict(head_stride=56), dict(head_stride=0), dict(token_stride=0), dict(token_stride=248), dict(head_stride=640, token_stride=56),
                dict(head_stride=632, token_stride=64), dict(head_stride=-56)):
        assert call(b, q_out=bad) == b.REC_ERR_ARG, bad


def test_more_than_a_launch_takes(b):
    assert call(b, heads=(1 << 20) - 1) == b.REC_ERR_OVERFLOW
    far = dict(token_stride=1 << 20, head_stride=64)
    assert call(b, tokens=1 << 31, heads=1, kv_heads=0, q_out=far) == b.REC_ERR_OVERFLOW
    assert call(b, tokens=(1 << 31) - 2000, heads=1, kv_heads=0, head_dim=128, q_out=far) == b.REC_ERR_OVERFLOW


def test_python_refuses_what_the_library_cannot_see(b):
    x, f = torch.zeros(10, 2, 64, dtype=torch.float16), torch.zeros(32, dtype=torch.float64)
    at = torch.zeros(10, dtype=torch.int32)
    for call in (lambda: b.rotate_heads(x, x, at, f), lambda: b.rotate_heads(None, None, at, f), lambda: b.rotate_heads(x[0], None, at, f),
                 lambda: b.rotate_heads(x.long(), None, at, f)):
        with pytest.raises(ValueError):
            call()


class OnDevice(torch.Tensor):
    """Host memory that says it is on device 0; a refused call looks at nothing more."""

    def get_device(self):
        return 0


def on(x):
    return x.as_subclass(OnDevice)


def test_python_refuses_tensors_that_do_not_fit(b, monkeypatch):
    monkeypatch.setattr(b, "_lib", None)
    x, f, at, w = on(torch.zeros(10, 2, 64)), on(torch.zeros(32, dtype=torch.float64)), on(torch.zeros(10, dtype=torch.int32)), on(torch.ones(64))
    bad = [dict(positions=at[:9]), dict(positions=at.float()), dict(positions=on(torch.zeros(20, dtype=torch.int32))[::2]), dict(positions=torch.zeros(10, dtype=torch.int32)),
           dict(frequencies=f.float()), dict(frequencies=f[None]), dict(frequencies=on(torch.zeros(64, dtype=torch.float64))[::2]),
           dict(q_weight=w.double()), dict(q_weight=w[:32]), dict(k_weight=on(torch.ones(128))[::2]), dict(k_weight=torch.ones(64)),
           dict(k=x[:9]), dict(k=x[..., :32]), dict(k=x.half()), dict(k=torch.zeros(10, 2, 64)), dict(k=on(torch.zeros(10, 2, 128))[..., ::2]),
           dict(q_out=x[:9]), dict(q_out=x.half()), dict(k_out=on(torch.zeros(10, 2, 128))[..., ::2]), dict(k=None, k_weight=w), dict(k=None, k_out=x),
           dict(q=on(torch.zeros(10, 2, 64, requires_grad=True))), dict(q_weight=on(torch.ones(64, requires_grad=True)))]
    for kw in bad:
        a = dict(q=x, k=x, positions=at, frequencies=f)
        a.update(kw)
        with pytest.raises(ValueError):
            b.rotate_heads(a.pop("q"), a.pop("k"), a.pop("positions"), a.pop("frequencies"), **a)


def bytes_of(r, tokens, heads, d, size):
    """Sets of 16-byte pieces that a rec_rows names."""
    return {(r.dev + size * (t * r.token_stride + h * r.head_stride)) // 16 + i for t in range(tokens) for h in range(heads) for i in range(d * size // 16)}


def places(tokens, heads, kv, d, size):
    """Ways to lay q, k, q_out and k_out out, as (q, k, q_out, k_out) of (offset in elements, token stride, head stride)."""
    far, all_ = 1 << 20, heads + 2 * kv
    row = all_ * d                                              # a projection's output: queries, keys, values of a token
    slices = ((0, row, d), (heads * d, row, d))
    apart = ((2 * far, heads * d, d), (3 * far, kv * d, d))
    yield *slices, *apart
    yield *slices, *slices                                      # in place
    yield *slices, slices[0], apart[1]
    yield *slices, slices[1], slices[0]                         # each in the other's
    yield *slices, slices[0], slices[0]
    yield *slices, ((heads + kv) * d, row, d), apart[1]         # among the values
    yield slices[0], slices[0], slices[0], apart[1]             # q is k, and gets its result first
    yield slices[0], slices[0], *apart
    by_three = ((0, 3 * heads * d, 3 * d), (d, 3 * heads * d, 3 * d))           # q, k and v of a head beside each other
    yield *by_three, *by_three
    yield *by_three, by_three[0], (2 * d, 3 * heads * d, 3 * d)
    yield *by_three, *reversed(by_three)
    by_head = ((0, d, tokens * d), (heads * tokens * d, d, tokens * d))         # heads before tokens
    yield *by_head, *by_head
    yield *by_head, by_head[0], (d, d, tokens * d)
    woven = ((0, 2 * d, 2 * tokens * d), (d, 2 * d, 2 * tokens * d))            # the same, q's tokens between k's
    yield *woven, *woven
    one = (heads * d, 0, d)                                                     # one token's keys for all, a projection's; one head's for all
    yield slices[0], one, slices[0], apart[1]
    yield slices[0], (d, 0, d), slices[0], apart[1]
    yield slices[0], (row * (tokens - 1) + heads * d, 0, 0), slices[0], apart[1]
    yield slices[0], (heads * d, row, 0), slices[0], apart[1]
    yield slices[0], (0, row, 0), slices[0], apart[1]
    for first in (0, d, 2 * d, 3 * d):                                          # heads two apart, three apart, and towards each other
        yield *apart, (0, 40 * d, 2 * d), (first, 40 * d, 3 * d)
        yield *apart, (0, -40 * d, 2 * d), (first, -40 * d, 3 * d)
        yield *apart, (0, 40 * d, 2 * d), (first + 8 * d, 40 * d, -2 * d)
        yield *apart, (0, 2 * d, 4 * tokens * d), (first, 2 * d, 6 * tokens * d)
    for shift in (16 // size, d, row, -row, heads * d - 16 // size, row * (tokens - 1), row * tokens, -row * tokens):
        yield slices[0], apart[1], (shift, row, d), (4 * far, kv * d, d)        # a result that lies a little further than q
        yield apart[0], slices[0], (shift, row, d), (5 * far, kv * d, d)
        yield *apart, (0, row, d), (shift, row, d)
        yield *apart, (0, -row, d), (shift, -row, d)
        yield *apart, (0, row, -d), (shift, row, -d)


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would run")
@pytest.mark.parametrize("tokens,heads,kv", [(1, 1, 1), (1, 3, 2), (2, 1, 1), (5, 4, 2), (7, 2, 2), (4, 1, 3), (9, 6, 1)])
@pytest.mark.parametrize("dtype,size,d", [(2, 2, 64), (0, 4, 32)])
def test_results_over_other_rows(b, tokens, heads, kv, dtype, size, d):
    """A result may be what it is made of, and nothing else that the call reads or writes: which was there first would be left to chance."""
    refused = allowed = 0
    for place in places(tokens, heads, kv, d, size):
        names, counts = ("q", "k", "q_out", "k_out"), (heads, kv, heads, kv)
        rows = {n: b.rec_rows((1 << 30) + size * at, token, head) for n, (at, token, head) in zip(names, place)}
        t = turn(b, tokens=tokens, heads=heads, kv_heads=kv, head_dim=d, pairs=0, dtype=dtype)
        for n in names:
            setattr(t, n, rows[n])
        held = {n: bytes_of(rows[n], tokens, c, d, size) for n, c in zip(names, counts)}
        clash = any(len(held[o]) < tokens * counts[names.index(o)] * d * size // 16 for o in ("q_out", "k_out")) or bool(held["q_out"] & held["k_out"])
        for o in ("q_out", "k_out"):
            for i in ("q", "k"):
                same = o[0] == i and rows[o].dev == rows[i].dev and (tokens == 1 or rows[o].token_stride == rows[i].token_stride) and \
                    (counts[names.index(o)] == 1 or rows[o].head_stride == rows[i].head_stride)
                clash |= not same and bool(held[o] & held[i])
        got = b._lib.rec_rotate_heads(C.byref(t), None)
        assert got == (b.REC_ERR_ARG if clash else b.REC_ERR_DEVICE), (place, clash)      # no device: further than its checks
        refused, allowed = refused + clash, allowed + (not clash)
    assert refused > 5 and allowed > 5


def test_results_between_rows_of_other_strides(b):
    """Where that cannot be told from the strides alone, rows between each other's count as overlapping."""
    base = dict(q=dict(dev=PTR), k=dict(dev=PTR + (1 << 24)), k_out=dict(dev=PTR + (1 << 25)))
    for bad in (dict(dev=PTR, token_stride=512), dict(dev=PTR + 128, token_stride=512, head_stride=128), dict(dev=PTR + (1 << 24), token_stride=320)):
        assert call(b, **base, q_out=bad) == b.REC_ERR_ARG, bad
    # as many pairs of heads as would take long to compare
    assert call(b, **{**base, "k_out": dict(dev=PTR + (1 << 30), token_stride=1 << 20, head_stride=192)}, heads=1 << 11, kv_heads=1 << 11,
                q_out=dict(dev=PTR + (1 << 30) + 128, token_stride=1 << 20, head_stride=128)) == b.REC_ERR_ARG
    huge = 1 << 60                      # spans that do not fit 64 bits
    assert call(b, **base, q_out=dict(dev=PTR, token_stride=huge, head_stride=huge >> 3)) == b.REC_ERR_ARG


def test_frequencies_that_require_grad(b, monkeypatch):
    """As queries, keys and weights do: their gradients would be lost without a word."""
    monkeypatch.setattr(b, "_lib", None)
    x, f, at = on(torch.zeros(10, 2, 64)), on(torch.zeros(32, dtype=torch.float64, requires_grad=True)), on(torch.zeros(10, dtype=torch.int32))
    with pytest.raises(ValueError, match="backward"):
        b.rotate_heads(x, x, at, f)
    with torch.no_grad(), pytest.raises(AttributeError):        # no library: further than the checks
        b.rotate_heads(x, x, at, f)
