"""rotate_heads() on the device, against its formulas in 64 bits (angles in 80) on the CPU."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32
HALF_STEP = {HF: 2.0 ** -11, BF: 2.0 ** -8, F32: 2.0 ** -24}
LEAST = {HF: 2.0 ** -25, BF: 2.0 ** -134, F32: 2.0 ** -150}       # half of the smallest number


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


def gen(seed):
    return torch.Generator().manual_seed(seed)


def frequencies(pairs, base=10000.0):
    return torch.from_numpy(base ** -(np.arange(pairs) / max(pairs, 1)))


def oracle(x, w, positions, f, eps, interleaved):
    """x [tokens, heads, D] -> (results, how far off each may be), float64.

    Counted: the result's rounding; of the row's norm the sum of D squares in fp32 (a chain of 16 and 4 exchanges, each half a
    step, halved by the root), its reciprocal root (a step) and two products: 2^-20 together; sines to four steps of fp32 with
    the angle's own rounding to fp32 turns (2 pi 2^-26): 2^-21; the angle in 64 bits: its product, its turns, and 1 / (2 pi) itself, half a step each."""
    d, pairs = x.shape[-1], len(f)
    y = x.double().numpy()
    with np.errstate(all="ignore"):
        if w is not None:
            y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps) * w.double().numpy()
        angle = positions.numpy().astype(np.longdouble)[:, None] * f.numpy().astype(np.longdouble)
        cos, sin = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
        a = np.arange(pairs) * (2 if interleaved else 1)
        z = a + (1 if interleaved else pairs)
        out, off = y.copy(), np.abs(y) * 2.0 ** -20
        out[..., a], out[..., z] = y[..., a] * cos - y[..., z] * sin, y[..., a] * sin + y[..., z] * cos
        size = np.abs(y[..., a]) + np.abs(y[..., z])
        off[..., a] = off[..., z] = size * (2.0 ** -20 + 2.0 ** -21 + 1.5 * 2.0 ** -52 * np.abs(angle).astype(np.float64)[:, None])
        off += np.abs(out) * HALF_STEP[x.dtype] + LEAST[x.dtype]
    return out, off


def close(got, want, off, what=""):
    got, (top, _) = got.double().cpu().numpy(), (torch.finfo(got.dtype).max, 0)
    assert got.shape == want.shape
    assert np.array_equal(np.isnan(got), np.isnan(want)), (what, np.argwhere(np.isnan(got) != np.isnan(want))[:5])
    fine = np.isfinite(want) & (np.abs(want) < top)
    bad = ~(np.abs(got[fine] - want[fine]) <= off[fine])
    assert not bad.any(), (what, int(bad.sum()), float(np.nanmax(np.abs(got[fine] - want[fine]) / off[fine])))


def check(b, q, k, positions, f, q_weight=None, k_weight=None, eps=1e-6, interleaved=False):
    cuda = lambda x: None if x is None else x.cuda()  # noqa: E731
    got = b.rotate_heads(cuda(q), cuda(k), cuda(positions), cuda(f), cuda(q_weight), cuda(k_weight), eps, interleaved)
    for x, w, y, name in ((q, q_weight, got[0], "q"), (k, k_weight, got[1], "k")):
        if x is None:
            assert y is None
            continue
        assert y.is_contiguous() and y.dtype is x.dtype
        close(y, *oracle(x, w, positions, f, eps, interleaved), name)


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("d,pairs", [(32, 16), (32, 8), (64, 32), (64, 8), (64, 24), (128, 64), (128, 40), (128, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_formula(b, dtype, d, pairs, interleaved):
    for tokens, heads, kv, seed in ((1, 1, 1, 1), (77, 3, 2, 2), (300, 8, 2, 3), (5, 33, 7, 4), (9, 1, 0, 5), (1100, 16, 8, 6), (4500, 1, 2, 7)):
        g = gen(seed)
        q, k = (torch.randn(tokens, h, d, generator=g).to(dtype) for h in (heads, kv))
        w = [1 + 0.3 * torch.randn(d, generator=g) for _ in range(2)]
        positions = torch.randint(-50, 5000, (tokens,), generator=g, dtype=torch.int32 if seed % 2 else torch.int64)
        check(b, q, k if kv else None, positions, frequencies(pairs), w[0] if seed != 3 else None, w[1] if kv and seed != 4 else None,
              interleaved=interleaved)


def test_only_keys_and_only_norms(b):
    g = gen(11)
    k, at = torch.randn(50, 2, 64, generator=g).to(BF), torch.arange(50)
    check(b, None, k, at, frequencies(32))
    check(b, k, None, at, frequencies(0), q_weight=torch.rand(64, generator=g))
    check(b, k, k, at, frequencies(0))


@pytest.mark.parametrize("dtype", [F32, BF])
def test_far_positions(b, dtype):
    """Times in seconds, the ends of int32, and counts past it: a sine in fp32 of an fp32 angle would be noise."""
    for at in (torch.tensor([2 ** 31 - 1, -2 ** 31, 1_700_000_000, 0, 1, -1], dtype=torch.int32),
               torch.tensor([2 ** 40, 2 ** 31, -2 ** 35 + 1, 1_700_000_000, 0, 7])):
        g = gen(12)
        q, k = (torch.randn(6, h, 64, generator=g).to(dtype) for h in (3, 1))
        check(b, q, k, at, frequencies(32), torch.ones(64), torch.ones(64))


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("eps", [1e-6, 0.0])
def test_rows_from_the_types_ends(b, dtype, eps):
    """Squares that overflow or vanish in fp32, zeros, and numbers that are not finite: their rows alone."""
    d, top = 64, torch.finfo(dtype).max
    x = torch.randn(16, 2, d, generator=gen(13))
    x[0] *= 1e30 if dtype is not HF else 1e4
    x[1] = top
    x[2] = torch.where(torch.arange(d) % 2 == 0, top, -top)
    x[3] *= 1e-30
    x[4] *= 1e-38
    x[5] = 0
    x[6, 0, 3] = float("inf")
    x[7, 1, 60] = float("nan")
    x[8, 0, :] = 0
    x[8, 0, 5] = 1e-25
    x[9] *= 1e18
    x[10] *= 1e-16
    x[11] = 0
    x[11, :, 63] = torch.finfo(dtype).tiny
    q = x.to(dtype)
    q = torch.where(torch.isinf(q) & torch.isfinite(x), torch.tensor(top, dtype=dtype), q)
    at = torch.arange(16)
    check(b, q, q.flip(0).contiguous(), at, frequencies(24), torch.ones(d), torch.full((d,), 0.5), eps=eps)
    check(b, q[3:], None, at[3:], frequencies(0), torch.ones(d), eps=eps)


def test_strided_rows_and_places(b):
    """Slices of a projection's rows; heads before tokens; results in place, and between rows that stay as they are."""
    g = gen(14)
    tokens, h, kv, d = 130, 6, 2, 64
    rows = torch.randn(tokens, h + 2 * kv, d, generator=g).to(BF)
    at, f, w = torch.randint(0, 1000, (tokens,), generator=g), frequencies(32), torch.rand(d, generator=g)
    check(b, rows[:, :h], rows[:, h:h + kv], at, f, w, w)
    by_head = torch.randn(h, tokens, d, generator=g).to(HF)
    check(b, by_head.transpose(0, 1), by_head.transpose(0, 1)[:, 1::2], at, f, w, w)
    check(b, rows[:, :1].expand(tokens, 3, d), rows[:1, :kv].expand(tokens, kv, d), at, f, w)      # one row for many heads or tokens
    live = rows.cuda()
    got = b.rotate_heads(live[:, :h], live[:, h:h + kv], at.cuda(), f.cuda(), w.cuda(), None, q_out=live[:, :h], k_out=live[:, h:h + kv])
    assert got[0].data_ptr() == live.data_ptr() and torch.equal(live[:, h + kv:].cpu(), rows[:, h + kv:])
    close(live[:, :h], *oracle(rows[:, :h], w, at, f, 1e-6, False))
    close(live[:, h:h + kv], *oracle(rows[:, h:h + kv], None, at, f, 1e-6, False))
    room = torch.full((h + 1, tokens + 2, d), 7.0, dtype=BF, device="cuda")
    b.rotate_heads(rows[:, :h].cuda(), None, at.cuda(), f.cuda(), w.cuda(), q_out=room[:h, 1:-1].transpose(0, 1))
    close(room[:h, 1:-1].transpose(0, 1), *oracle(rows[:, :h], w, at, f, 1e-6, False))
    assert (room[h] == 7).all() and (room[:, 0] == 7).all() and (room[:, -1] == 7).all()


def test_empty_calls(b):
    f = frequencies(32).cuda()
    q, k = b.rotate_heads(torch.zeros(0, 4, 64, device="cuda"), torch.zeros(0, 2, 64, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"), f)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    q, k = b.rotate_heads(torch.zeros(5, 0, 64, device="cuda"), None, torch.zeros(5, dtype=torch.int32, device="cuda"), f)
    assert q.shape == (5, 0, 64)


def test_in_a_graph_and_on_another_stream(b):
    g = gen(15)
    q = torch.randn(200, 4, 64, generator=g).to(BF).cuda()
    at, f, w, out = torch.arange(200).cuda(), frequencies(32).cuda(), torch.rand(64, generator=g).cuda(), torch.empty_like(q)
    b.rotate_heads(q, None, at, f, w, q_out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.rotate_heads(q, None, at, f, w, q_out=out)
    for _ in range(3):
        q.copy_(torch.randn(200, 4, 64, generator=g).to(BF))
        at += 91
        graph.replay()
        eager, _ = b.rotate_heads(q, None, at, f, w)
        assert torch.equal(out, eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there, _ = b.rotate_heads(q, None, at, f, w)
    side.synchronize()
    assert torch.equal(there, eager)
