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
