"""Attention over cached histories in the forms that a launch takes by its size (two kv heads a wave,
one wave a block, parts of a history in one wave), pages behind 2^32 bytes, and rows that are computed again."""
import numpy as np
import pytest
import torch

import history_oracle as O
from test_gpu_history import BF, HF, F32, Histories, gen, whole, expect_whole

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


def check_some(s, q, got, picks, scale, window=0, sinks=0, candidates=False, what=""):
    """Histories `picks` of a call against the oracle."""
    qn = q.double().cpu().numpy()
    _, nq, heads, d = qn.shape
    per = heads // s.kv
    for i in picks:
        n = s.lengths[i]
        at = [n - 1 if candidates else n - nq + x for x in range(nq)]
        want, off = np.zeros(qn.shape[1:]), np.zeros(qn.shape[1:])
        for h in range(heads):
            k, v = (x[s.ends[i]:s.ends[i + 1], h // per] for x in (s.k, s.v))
            want[:, h], off[:, h] = O.attend_rows(qn[i, :, h], k, v, at, scale, window, sinks, q.dtype)
        O.assert_close(got[i], want, off, (what, i, n))


def many_lengths(batch, most, seed):
    n = torch.randint(0, most + 1, (batch,), generator=gen(seed)).tolist()
    n[:6] = [0, 1, 2, most, 64, 65][:6]
    return [min(x, most) for x in n]


@pytest.mark.parametrize("d,kv,per,queries,fmt,dtype", [
    (32, 2, 2, 1, "mx8", HF), (32, 4, 1, 3, "mx4", BF), (64, 2, 8, 1, "mx4", BF), (64, 2, 3, 2, "mx8", HF), (32, 2, 4, 2, "mx4", HF),  # two heads a wave
    (64, 2, 9, 1, "mx4", BF), (64, 3, 2, 1, "mx8", BF), (128, 2, 2, 1, "mx4", HF), (128, 2, 1, 2, "mx8", BF), (32, 3, 1, 1, "mx4", BF)])  # one
def test_many_histories(b, d, kv, per, queries, fmt, dtype):
    """At least 4096 pairs of history and head."""
    batch = -(-4100 // kv)
    s = Histories(b, many_lengths(batch, 140, d + kv), kv, d, fmt, 32, seed=40)
    q = torch.randn(batch, queries, kv * per, d, generator=gen(41)).to(dtype).cuda()
    picks = list(range(8)) + list(range(8, batch, 211)) + [batch - 1]
    for window, sinks, candidates in ((0, 0, False), (9, 2, False), (70, 0, True)):
        got = s.cache.attend(q, s.table, s.len_t, window=window, sinks=sinks, candidates=candidates)
        check_some(s, q, got, picks, d ** -0.5, window, sinks, candidates, (window, sinks))
    assert s.cache.check()[0] == b.REC_OK


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
def test_many_histories_ignore_what_they_do_not_see(b, fmt):
    """NaN in one head's keys and values of some histories: two heads share a wave, and only one of them shows it."""
    batch, kv, d, n, window, sinks = 2060, 2, 64, 100, 30, 2
    s = Histories(b, [n] * batch, kv, d, fmt, 32, seed=42)
    q = torch.randn(batch, 2, 4, d, generator=gen(43)).to(BF).cuda()
    bad = {3: 1, 4: 50, 5: 69, 6: 70, 7: 98, 8: 99}       # seen by both queries, neither, the first, both, both, the second
    rows = torch.tensor([s.ends[i] + j for i, j in bad.items()])
    k, v = (torch.from_numpy(x[rows.numpy()]).float() for x in (s.k, s.v))
    k[:, 1] = v[:, 1] = float("nan")
    s.cache.write(k.cuda(), v.cuda(), s.slots[rows].cuda())
    assert s.cache.check()[0] == b.REC_ERR_VALUE
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    got = s.cache.attend(q, s.table, s.len_t, window=window, sinks=sinks)
    check_some(s, q, got, [0, 1, 2, *bad, 9, 10, batch - 1], d ** -0.5, window, sinks)
    assert not got[4].isnan().any() and got[7, :, 2:].isnan().all() and not got[:, :, :2].isnan().any()


def test_parts_of_one_wave(b):
    """2048 pairs: blocks of one wave, whose histories are still divided."""
    batch, d = 1024, 64
    s = Histories(b, many_lengths(batch, 300, 1), 2, d, "mx4", 64, seed=44, width=16)
    q = torch.randn(batch, 1, 4, d, generator=gen(45)).to(BF).cuda()
    for window, sinks in ((0, 0), (200, 4)):
        got = s.cache.attend(q, s.table, s.len_t, window=window, sinks=sinks)
        check_some(s, q, got, [*range(8), *range(8, batch, 97)], d ** -0.5, window, sinks, what=window)


@pytest.mark.parametrize("fmt,d", [("mx4", 128), ("mx8", 64)])
def test_pages_behind_four_gigabytes(b, fmt, d):
    """The first and the last pages of a cache of more than 2^32 bytes."""
    kv, page_tokens = 8, 256
    per_page = kv * page_tokens * d * (17 if fmt == "mx4" else 33) // 16
    pages = (2 ** 32 + 2 ** 28) // per_page + 1
    cache = b.HistoryCache(pages, page_tokens, kv, d, fmt)
    assert cache.pages.numel() > 2 ** 32
    mine = torch.tensor([0, pages - 1, 1, pages - 2])
    cache.pages[mine.cuda()] = 255
    n = 4 * page_tokens - 30
    at = torch.arange(n)
    slots = mine[at // page_tokens] * page_tokens + at % page_tokens
    k, v = (torch.randn(n, kv, d, generator=gen(i)) for i in (1, 2))
    cache.write(k.cuda(), v.cuda(), slots.cuda())
    small = b.HistoryCache(4, page_tokens, kv, d, fmt)
    small.pages.fill_(255)
    small.write(k.cuda(), v.cuda(), at.cuda())
    assert torch.equal(cache.pages[mine.cuda()], small.pages)
    for x, y in zip(cache.read(slots.cuda(), F32), small.read(at.cuda(), F32)):
        assert torch.equal(x, y)
    q = torch.randn(1, 1, 2 * kv, d, generator=gen(3)).to(BF).cuda()
    length = torch.tensor([n], dtype=torch.int32).cuda()
    got = cache.attend(q, mine[None].int().cuda(), length)
    assert torch.equal(got, small.attend(q, torch.arange(4, dtype=torch.int32)[None].cuda(), length))
    assert cache.check()[0] == small.check()[0] == b.REC_OK


def test_a_row_computed_again_has_no_weight_on_scores_of_minus_infinity(b):
    """Values that are NaN behind a row make it be computed again; its first 64 scores are -inf, later ones finite."""
    lengths, d = [100], 32
    q, k, v, offsets = whole(lengths, 1, 1, d, BF, 46, fused=False)
    q.fill_(3.0e38)
    k[:70] = -1.0e38
    k[70:] = 0.0
    v[95] = float("nan")
    v[0, 0, 3] = float("nan")                # under a weight of zero: 0 * NaN
    got = b.attend_window(q, k, v, offsets, scale=1.0, window=90, sinks=0).double().cpu().numpy()
    values = v.double().cpu().numpy()
    for row in (71, 80, 89, 92, 94):
        want = values[70:row + 1, 0].mean(0)
        if row - 90 < 0:
            want[3] = np.nan
        fine = np.isfinite(want)
        assert np.array_equal(np.isfinite(got[row, 0]), fine), row
        # the sum's weights are exact; the mean is rounded once, and once more in sums of at most 25 terms in fp32
        assert (np.abs(got[row, 0] - want)[fine] <= 2.0 ** -8 * np.abs(want)[fine] + 2.0 ** -20).all(), row
    assert np.isnan(got[:70]).all() and np.isnan(got[95:]).all()


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("dtype,d", [(BF, 32), (HF, 64), (F32, 128), (F32, 64)])
def test_every_16_bit_number_is_stored_nearest(b, fmt, dtype, d):
    """Each finite bf16 or fp16 number as a block's largest, beside numbers up to its size; fp32 the same with lower bits."""
    g = gen(47)
    bits = torch.arange(0, 2 ** 15, 7, dtype=torch.int32)
    top = bits.to(torch.int16).view(HF if dtype == HF else BF).float()
    top = top[torch.isfinite(top)]
    if dtype == F32:
        top = torch.cat((top * (1 - 2.0 ** -10 * torch.rand(top.shape, generator=g)), torch.tensor([3.4028234e38, 1.8125 * 2.0 ** 127, 1.75 * 2.0 ** 127])))
    x = top[:, None] * (2 * torch.rand(len(top), d, generator=g) - 1)
    x[:, ::32] = top[:, None]
    x = x.to(dtype)[:, None]
    n = len(x)
    c = b.HistoryCache(-(-n // 64), 64, 1, d, fmt)
    slots = torch.arange(n).cuda()
    c.write(x.cuda(), x.flip(2).contiguous().cuda(), slots)
    assert c.check()[0] == b.REC_OK
    rk, rv = c.read(slots, F32)
    codes, scales = O.quantise(x.double().numpy().reshape(-1, 32), fmt)
    want = torch.from_numpy(O.values(codes, fmt) * O.scale_values(scales)[:, None]).view(n, 1, d)
    assert torch.equal(rk.cpu().double(), want) and torch.equal(rv.cpu().double(), want.flip(2))


@pytest.mark.parametrize("batch,width,most,long", [(1024, 8, 300, ()), (1100, 70, 90, (4400, 2000, 2100)), (2100, 20, 90, (1200,)), (4200, 20, 60, (1000, 1279))])
def test_a_few_much_longer_than_most(b, batch, width, most, long):
    """Blocks of one wave whose histories are divided; of four, with parts and without; and more pairs than those are for."""
    d = 64
    n = many_lengths(batch, most, 2)
    n[6:6 + len(long)] = long
    s = Histories(b, n, 2, d, "mx4", 64, seed=48, width=width)
    q = torch.randn(batch, 1, 4, d, generator=gen(49)).to(BF).cuda()
    for window, sinks in ((0, 0), (70, 4)):
        got = s.cache.attend(q, s.table, s.len_t, window=window, sinks=sinks)
        check_some(s, q, got, [*range(10), *range(10, batch, 211)], d ** -0.5, window, sinks, what=window)
    assert s.cache.check()[0] == b.REC_OK
