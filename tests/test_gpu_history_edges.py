"""User histories at the edges of their contract: what a row does not see, whatever it holds."""
import numpy as np
import pytest
import torch

import history_oracle as O
from test_gpu_history_forms import check_some, many_lengths
from test_gpu_history import BF, HF, F32, Histories, expect_whole, gen, whole

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


# ------------------------------------------------------------ codes that are NaN
def poke_value(s, row, head, column, byte):
    """Sets the code of one column of a stored value (mx8), under the scale that is there."""
    page, at = divmod(int(s.slots[row]), s.page_tokens)
    block, j = divmod(column, 32)
    d = s.d
    place = 16 * d + ((16 * block + j % 16) * 16 + at % 16) * 2 + j // 16
    s.cache.pages[page, head, at // 16, place] = byte


@pytest.mark.parametrize("d,kv,per,dtype", [(32, 2, 1, HF), (64, 1, 4, BF), (128, 2, 2, BF), (128, 1, 3, HF)])
@pytest.mark.parametrize("batch", [1, 2060])           # few pairs; enough for two kv heads a wave
def test_a_code_that_is_nan_reaches_only_the_rows_that_see_it(b, d, kv, per, dtype, batch):
    """E4M3 has codes that are NaN under any scale.  No call stores one, but a place that was never written may hold
    it, and a length may count that place."""
    n, nq, window, sinks = 100, 5, 40, 2
    if batch > 1 and d == 128:
        batch = 40
    # For each history a token, the column and the head: seen by some queries, by none, by all; first of a window, last token.
    where = [(98, 0), (97, d - 1), (99, 17), (57, 5), (58, 16), (60, d // 2), (30, 3), (1, 20), (2, 9), (70, 31)]
    for shift in range(len(where) if batch == 1 else 1):
        s = Histories(b, [n] * batch, kv, d, "mx8", 32, seed=51)
        q = torch.randn(batch, nq, kv * per, d, generator=gen(52)).to(dtype).cuda()
        at = {i: where[(i + shift) % len(where)] for i in range(min(batch, len(where)))}
        for i, (token, column) in at.items():
            poke_value(s, int(s.ends[i]) + token, i % kv, column, 0x7f if i % 2 else 0xff)
        s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
        for (token, column), i in zip(at.values(), at):
            assert np.isnan(s.v[s.ends[i] + token, i % kv, column])
        got = s.cache.attend(q, s.table, s.len_t, window=window, sinks=sinks)
        qn = q.double().cpu().numpy()
        for i in [*at, batch - 1]:
            want, off = np.zeros(qn.shape[1:]), np.zeros(qn.shape[1:])
            for h in range(kv * per):
                k, v = (x[s.ends[i]:s.ends[i + 1], h // per] for x in (s.k, s.v))
                want[:, h], off[:, h] = O.attend_rows(qn[i, :, h], k, v, range(n - nq, n), d ** -0.5, window, sinks, dtype)
            if i in at:     # one column of the rows that see the token, and of the heads that share the kv head
                token, column = at[i]
                for x in range(nq):
                    sees = O.sees(n - nq + x, token, window, sinks)
                    assert np.isnan(want[x]).sum() == (per if sees else 0), (i, token, x)
            O.assert_close(got[i], want, off, (i, at.get(i)))


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("fill", [0x7f, 0x7e])
def test_places_within_a_length_that_were_never_written(b, d, fill):
    """The last two tokens of each history were left out of the write: earlier queries are as if they were not there."""
    n, nq = 70, 4
    s = Histories(b, [n, n], 1, d, "mx8", 32, seed=53)
    k, v = s.cache.read(s.slots.cuda(), F32)
    s.cache.pages.fill_(fill)
    slots = s.slots.clone()
    for e in s.ends[1:]:
        slots[e - 2:e] = -1
    s.cache.write(k, v, slots.cuda())
    q = torch.randn(2, nq, 2, d, generator=gen(54)).to(BF).cuda()
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    want, off = s.expect(q, d ** -0.5, 0, 0, False)
    assert np.isfinite(want[:, :2]).all() and (fill != 0x7f or np.isnan(want[:, 2:]).all())
    O.assert_close(s.cache.attend(q, s.table, s.len_t), want, off)


# ------------------------------------------------------------------- scale of zero
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_a_query_that_is_not_finite_has_no_result_under_a_scale_of_zero(b, dtype, d):
    """0 * inf is NaN: in whole histories and over the cache; other rows get the mean of what they see."""
    n, heads = 45, 2
    q, k, v = (torch.randn(n, h, d, generator=gen(60 + h)).to(dtype) for h in (heads, 1, 1))
    bad = {(0, 0): float("inf"), (7, 1): float("nan"), (31, 0): float("-inf"), (44, 1): float("inf")}
    for i, ((row, head), x) in enumerate(bad.items()):
        q[row, head, (5 * i) % d] = x
    q[20, 0] = torch.finfo(dtype).max              # large, and finite
    q, k, v = q.cuda(), k.cuda(), v.cuda()
    vn = v.double().cpu().numpy()[:, 0]
    want, off = np.zeros((n, heads, d)), np.zeros((n, heads, d))
    for row in range(n):
        for head in range(heads):
            want[row, head] = np.nan if (row, head) in bad else vn[:row + 1].mean(0)
            # weights and the mean are rounded to the type
            off[row, head] = O.EPS[dtype] * (np.abs(want[row, head]) + np.abs(vn[:row + 1]).mean(0)) + 2.0 ** -20
    O.assert_close(b.attend_window(q, k, v, torch.tensor([0, n], dtype=torch.int32).cuda(), scale=0.0), want, off)

    cache = b.HistoryCache(2, 32, 1, d, "mx8")
    slots = torch.arange(n).cuda()
    cache.write(k, v, slots)
    vn = cache.read(slots, F32)[1].double().cpu().numpy()[:, 0]
    for row in range(n):
        for head in range(heads):
            want[row, head] = np.nan if (row, head) in bad else vn[:row + 1].mean(0)
            off[row, head] = O.EPS[dtype] * (np.abs(want[row, head]) + np.abs(vn[:row + 1]).mean(0)) + 2.0 ** -20
    got = cache.attend(q[None], torch.arange(2, dtype=torch.int32)[None].cuda(), torch.tensor([n], dtype=torch.int32).cuda(), scale=0.0)
    O.assert_close(got[0], want, off)


# ------------------------------------------------- small weights beside a large one
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("below", [10.0, 14.0, 17.5, 20.0])
@pytest.mark.parametrize("first", [True, False])
def test_many_small_weights_beside_a_large_one(b, dtype, d, below, first):
    """One key is e^below more likely than each of 4000 others, and its value is zero, so that the others are the result.
    A weight is its type's rounding of itself, or off by at most 2^-36 of the largest (fp16 ends where bf16 and fp32 go on)."""
    n = 4001
    q, k, v = torch.zeros(n, 1, d), torch.zeros(n, 1, d), torch.rand(n, 1, d, generator=gen(61)) + 0.5
    at = 0 if first else n - 3
    q[:, 0, 3], k[at, 0, 3], v[at] = 4.0, below / 4, 0.0
    q, k, v = (x.to(dtype).cuda() for x in (q, k, v))
    got = b.attend_window(q, k, v, torch.tensor([0, n], dtype=torch.int32).cuda(), scale=1.0)
    rows = [at + 1, at + 2, n - 2, n - 1] if not first else [1, 63, 64, 65, 1000, n - 1]
    qn, kn, vn = (x.double().cpu().numpy()[:, 0] for x in (q, k, v))
    want, off = O.attend_rows(qn[rows], kn, vn, rows, 1.0, 0, 0, dtype)
    if dtype == HF:
        off += np.array(rows)[:, None] * 2.0 ** -36 * np.abs(vn).max()
    O.assert_close(got[rows, 0], want, off)


# ------------------------------------------------------------------- fault records
def test_fault_records_that_have_words_between(b):
    """Refused: kernels write four adjacent words."""
    q = torch.zeros(4, 1, 32, dtype=BF, device="cuda")
    offsets = torch.tensor([0, 4], dtype=torch.int32).cuda()
    words = torch.full((16,), -1, dtype=torch.int64, device="cuda")
    for fault in (words[::2], words[:3], words.int()):
        with pytest.raises(ValueError):
            b.attend_window(q, q, q, offsets, fault=fault)
        with pytest.raises(ValueError):
            b.rec_history_check(fault)
    b.attend_window(q, q, q, offsets, fault=words[4:8])
    assert b.rec_history_check(words[4:8]) == (b.REC_OK, -1, -1) and bool((words == -1).all())


def test_a_fault_that_comes_while_a_record_is_checked_stays(b):
    """A check clears what it read: a word that another stream has lowered since is the next check's."""
    record = torch.tensor([5, -1, 7, 9], dtype=torch.int64).cuda()
    assert b.rec_probe_clear_faults(record, [5, -1, 8, 9]) == b.REC_OK
    assert record.tolist() == [-1, -1, 7, -1]
    assert b.rec_probe_clear_faults(record, [-1, -1, -1, -1]) == b.REC_OK      # read before there was any
    assert record.tolist() == [-1, -1, 7, -1]
    assert b.rec_history_check(record) == (b.REC_ERR_INDEX_RANGE, 7, b.REC_FAULT_PAGE)
    assert b.rec_history_check(record) == (b.REC_OK, -1, -1)


# ------------------------------------------------------- rows that are computed again
@pytest.mark.parametrize("d,dtype", [(32, HF), (32, BF), (64, BF), (64, HF), (128, BF), (128, HF)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 3), (100, 0), (37, 5), (64, 64), (30, 200), (257, 1)])
def test_rows_beside_numbers_that_are_not_finite(b, d, dtype, window, sinks):
    """Rows that see them, in a column or in all, and rows of the same tiles that do not."""
    lengths = [300, 1, 64]
    q, k, v, offsets = whole(lengths, 4, 2, d, dtype, 70)
    v[2, 0, 5] = float("nan")
    v[130, 1, d - 1] = float("inf")
    v[131, 1, d - 1] = float("-inf")
    v[200, 0] = float("nan")
    k[250, 1, 7] = float("nan")
    q[290, 3, 0] = float("inf")
    k[300, 0, 0] = float("-inf")
    v[301 + 20, 1] = float("inf")
    want, off = expect_whole(q, k, v, lengths, d ** -0.5, window, sinks)
    got = b.attend_window(q, k, v, offsets, window=window, sinks=sinks)
    gn = got.double().cpu().numpy()
    assert np.array_equal(np.isposinf(gn), np.isposinf(want)) and np.array_equal(np.isneginf(gn), np.isneginf(want))
    O.assert_close(got, want, off)


# --------------------------------------------------- values next to the range's end
@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("lengths,kv,per,d", [([200, 3], 1, 2, 64), ([5000], 2, 1, 128), ([90] * 2060, 2, 2, 32)])
def test_means_of_the_largest_values(b, fmt, lengths, kv, per, d):
    """A mean of values up to 2^128 is no larger than they are; their sum is.  One wave, several, parts, two heads a wave."""
    s = Histories(b, lengths, kv, d, fmt, 32, seed=80)
    g = gen(81)
    v = torch.sign(torch.randn(1, kv, d, generator=g)) * 2.0 ** 127 * (1 + 0.75 * torch.rand(len(s.slots), kv, d, generator=g))
    k = torch.from_numpy(s.k).float()
    s.cache.write(k.cuda(), v.cuda(), s.slots.cuda())
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    assert np.abs(s.v).max() > 2.5e38 and np.isfinite(s.v).all()
    q = torch.randn(len(lengths), 1, kv * per, d, generator=g).to(BF).cuda()
    got = s.cache.attend(q, s.table, s.len_t)
    qn = q.double().cpu().numpy()
    for i in sorted({0, len(lengths) // 2, len(lengths) - 1}):
        for h in range(kv * per):
            kk, vv = (x[s.ends[i]:s.ends[i + 1], h // per] for x in (s.k, s.v))
            want, off = O.attend_rows(qn[i, :, h], kk, vv, [lengths[i] - 1], d ** -0.5, 0, 0, BF)
            O.assert_close(got[i, :, h], want, off, (i, h))


@pytest.mark.parametrize("d", [32, 64, 128])
def test_means_of_the_largest_values_in_whole_histories(b, d):
    q, k, v, offsets = whole([150, 1, 40], 2, 1, d, BF, 82, fused=False)
    v = (torch.sign(v[:1].float()) * 2.0 ** 127 * (1 + 0.9 * torch.rand(v.shape, generator=gen(83)).cuda())).to(BF)
    for window, sinks in ((0, 0), (20, 3)):
        O.assert_close(b.attend_window(q, k, v, offsets, window=window, sinks=sinks), *expect_whole(q, k, v, [150, 1, 40], d ** -0.5, window, sinks))


# ------------------------------------------------------------- forms, as they are taken
@pytest.mark.parametrize("form,batch,width,most,long,kv,d,fmt,dtype,queries", [
    ((1, 2, 1), 1024, 8, 500, (512,), 2, 64, "mx4", BF, 1),               # a wave a block, two parts
    ((1, 2, 1), 1024, 8, 500, (512, 511), 2, 32, "mx8", HF, 3),
    ((1, 1, 1), 2048, 2, 128, (), 2, 128, "mx8", BF, 1),                  # a wave for all of a history
    ((2, 1, 1), 700, 8, 400, (512,), 2, 64, "mx8", HF, 2),                # two waves
    ((2, 2, 1), 512, 8, 500, (512, 449), 2, 64, "mx4", BF, 1),            # in two parts
    ((4, 1, 1), 300, 4, 256, (), 2, 128, "mx4", HF, 2),                   # four
    ((4, 2, 1), 1100, 75, 90, (4800, 2000, 2100), 2, 64, "mx4", BF, 1),   # in parts, for the few long ones
    ((4, 16, 1), 8, 128, 3000, (8192, 8191), 2, 64, "mx4", HF, 18),        # in as many as work at once
    ((1, 1, 2), 4200, 4, 200, (256,), 2, 64, "mx8", BF, 2)])              # two kv heads a wave
def test_forms_by_size(b, form, batch, width, most, long, kv, d, fmt, dtype, queries):
    n = many_lengths(batch, most, 3)
    n[6:6 + len(long)] = long[:max(0, len(n) - 6)]
    n = n[:batch]
    s = Histories(b, n, kv, d, fmt, 64, seed=90, width=width)
    q = torch.randn(batch, queries, 2 * kv, d, generator=gen(91)).to(dtype).cuda()
    for window, sinks in ((0, 0), (150, 3)):
        query = b.rec_query(q.data_ptr(), q.data_ptr(), *q.stride()[:3], b._ATTEND_CODES[dtype], batch, queries, 2 * kv, s.table.data_ptr(),
                            s.table.stride(0), width, s.len_t.data_ptr(), 1.0, window, sinks, 0)
        if not window:
            assert b.rec_probe_history_form(s.cache._h, query) == (b.REC_OK, *form)
        got = s.cache.attend(q, s.table, s.len_t, window=window, sinks=sinks)
        check_some(s, q, got, sorted({*range(min(batch, 9)), *range(9, batch, 211)}), d ** -0.5, window, sinks, what=(window, sinks))
    assert s.cache.check()[0] == b.REC_OK


# --------------------------------------------------------- nothing outside the buffers
def guarded(rows, columns, dtype, margin=64):
    """A buffer of rows with `margin` more on both sides, all of one pattern, and the rows by themselves."""
    whole = torch.full((rows + 2 * margin, columns), 0x5A, dtype=torch.uint8, device="cuda").repeat_interleave(torch.finfo(dtype).bits // 8, 1)
    return whole, whole[margin:margin + rows].view(dtype)


def untouched(whole, rows, margin=64):
    return bool((whole[:margin] == 0x5A).all()) and bool((whole[margin + rows:] == 0x5A).all())


@pytest.mark.parametrize("offsets", [[0, 20, 20, 50], [0, 30, 20, 50], [0, 10, 60, 50], [-5, 10, 20, 50], [5, 10, 20, 50], [0, 10, 20, 49], [0, 10, 20, 5000],
                                     [50, 0, 50, 0], [-2 ** 31, 2 ** 31 - 1, -1, 50], [0, 50, 50, 50]])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_outputs_of_whole_histories_stay_within_their_buffer(b, offsets, d):
    heads, n = 2, 50
    q, k, v, _ = whole([n], heads, 1, d, BF, 95, fused=False)
    buffer, out = guarded(n, heads * d, BF)
    fault, at = b._faults("cuda:0"), torch.tensor(offsets, dtype=torch.int32).cuda()
    r = lambda t: b.rec_rows(t.data_ptr(), t.stride(0), t.stride(1))  # noqa: E731
    w = b.rec_window(r(q), r(k), r(v), out.data_ptr(), b.REC_BF16, len(offsets) - 1, n, heads, 1, d, at.data_ptr(), d ** -0.5, 0, 0, fault.data_ptr())
    assert b.rec_window_attend(w) == b.REC_OK
    torch.cuda.synchronize()
    assert untouched(buffer, n)
    good = offsets in ([0, 20, 20, 50], [0, 50, 50, 50])
    assert (b.rec_history_check(fault)[0] == b.REC_OK) == good
    if good:
        lengths = [y - x for x, y in zip(offsets, offsets[1:])]
        O.assert_close(out.view(n, heads, d), *expect_whole(q, k, v, lengths, d ** -0.5, 0, 0))


@pytest.mark.parametrize("lengths,queries,width", [([1, 0, 40], 1, 4), ([100, 7, 64], 5, 4), ([3000], 1, 100), ([9, -4, 10 ** 6], 3, 4)])
def test_outputs_over_the_cache_stay_within_their_buffer(b, lengths, queries, width):
    """One wave, several rows, parts; lengths that are none."""
    d, heads = 64, 2
    s = Histories(b, [max(0, min(n, 32 * width)) for n in lengths], 1, d, "mx8", 32, seed=96, width=width)
    q = torch.randn(len(lengths), queries, heads, d, generator=gen(97)).to(BF).cuda()
    rows = len(lengths) * queries * heads
    buffer, out = guarded(rows, d, BF)
    s.cache.attend(q, s.table, torch.tensor(lengths, dtype=torch.int32).cuda(), out=out.view(q.shape))
    torch.cuda.synchronize()
    assert untouched(buffer, rows)
    want, off = s.expect(q, d ** -0.5, 0, 0, False)
    O.assert_close(out.view(q.shape), want, off)


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_a_write_touches_its_slots_and_nothing_else(b, fmt, d):
    """Every byte of places that are not named stays: whole groups, parts of groups, single slots."""
    kv, pages, page_tokens = 2, 6, 32
    cache = b.HistoryCache(pages, page_tokens, kv, d, fmt)
    slots = torch.cat((torch.arange(32, 55), torch.tensor([3, 100, -1, 101, 191]), torch.arange(128, 160)))
    k, v = (torch.randn(len(slots), kv, d, generator=gen(98 + i)).cuda() for i in range(2))
    raw = {}
    for fill in (0x00, 0xff, 0xa5):
        cache.pages.fill_(fill)
        cache.write(k, v, slots.cuda())
        raw[fill] = cache.pages.cpu().numpy()
    same = (raw[0x00] == raw[0xff]) & (raw[0x00] == raw[0xa5])         # written: the same bytes whatever was there
    kept = (raw[0x00] == 0x00) & (raw[0xff] == 0xff) & (raw[0xa5] == 0xa5)
    assert (same | kept).all() and not (same & kept).any()
    named = int((slots >= 0).sum())
    assert int(same.sum()) == named * kv * d * (17 if fmt == "mx4" else 33) // 16
    ours = {int(x) // 16 for x in slots if x >= 0}
    for group in range(pages * page_tokens // 16):
        page, g = divmod(group, page_tokens // 16)
        assert same[page, :, g].any() == (group in ours)


# ---------------------------------------------------------- how exactly a query is held
@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("dtype,bits", [(BF, 8), (BF, 13), (BF, 16), (HF, 8), (HF, 13)])
def test_small_elements_of_a_query_beside_a_large_one(b, fmt, d, dtype, bits):
    """A score that is one small element alone, 2^-bits of the largest of its 32, which meets zeros.  A query's terms end at half of
    2^-13 (fp16: 2^-17) where its largest is at least 224, so that the score is off by that; besides, the weight's and the output's rounding."""
    batch, heads = 40, 4
    g = gen(100 + bits)
    column = torch.randint(0, d, (batch,), generator=g)
    beside = column // 32 * 32 + (column + 1 + torch.randint(0, 31, (batch,), generator=g)) % 32
    beside = torch.where(beside == column, column // 32 * 32 + (column + 1) % 32, beside)
    top = 2.0 ** (10 if dtype == HF else 20)
    q = (1 + torch.rand(batch, heads, d, generator=g)) * top * 2.0 ** -bits
    q[torch.arange(batch), :, beside] = top * (1 + torch.rand(batch, heads, generator=g))
    q = q.to(dtype)
    k = torch.zeros(2 * batch, 1, d)
    k[1::2, 0][torch.arange(batch), column] = 1.0
    v = torch.zeros(2 * batch, 1, d)
    v[1::2] = torch.randn(batch, 1, d, generator=g)
    cache = b.HistoryCache(batch, 16, 1, d, fmt)
    slots = (torch.arange(batch)[:, None] * 16 + torch.arange(2)).reshape(-1).cuda()
    cache.write(k.cuda(), v.cuda(), slots)
    v = cache.read(slots, F32)[1].cpu().double().numpy()[1::2, 0]
    scale = 2.0 ** bits / top
    got = cache.attend(q.cuda(), torch.arange(batch, dtype=torch.int32)[:, None].cuda(), torch.full((batch,), 2, dtype=torch.int32).cuda(), scale=scale)
    qn = q.double().numpy()
    x = qn[np.arange(batch), :, column.numpy()] * scale                                    # [batch, heads]
    want = (1 / (1 + np.exp(-x)))[..., None] * v[:, None]
    largest = np.abs(qn).max(-1)
    score = scale * largest * (2.0 ** -14 if dtype == BF else 2.0 ** -18) / 224 + np.abs(x) * (d + 8) * 2.0 ** -24
    off = (2 * O.EPS[dtype] + 2 * score[..., None] + 2.0 ** -20) * np.abs(want) + 2.0 ** -25
    O.assert_close(got, want, off)


# --------------------------------------------------------- scales that no write makes
@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_infinite_places_within_a_length_that_were_never_written(b, fmt, d):
    """Bytes of 254: the largest codes under a scale of 2^127, beyond fp32."""
    n, nq = 70, 4
    s = Histories(b, [n, n], 1, d, fmt, 32, seed=55)
    k, v = s.cache.read(s.slots.cuda(), F32)
    s.cache.pages.fill_(254)
    slots = s.slots.clone()
    for e in s.ends[1:]:
        slots[e - 2:e] = -1
    s.cache.write(k, v, slots.cuda())
    q = torch.randn(2, nq, 2, d, generator=gen(56)).to(BF).cuda()
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    assert np.isinf(s.v[s.ends[1] - 1]).all()
    want, off = s.expect(q, d ** -0.5, 0, 0, False)
    assert np.isfinite(want[:, :2]).all() and np.isnan(want[:, 2:]).all()
    O.assert_close(s.cache.attend(q, s.table, s.len_t), want, off)


@pytest.mark.parametrize("fmt,byte", [("mx4", 253), ("mx4", 254), ("mx8", 247), ("mx8", 254)])
@pytest.mark.parametrize("d,kv,per,dtype", [(32, 2, 1, HF), (64, 1, 4, BF), (128, 2, 2, BF)])
@pytest.mark.parametrize("batch", [10, 2060])
def test_a_value_under_a_scale_that_no_write_makes_reaches_only_the_rows_that_see_it(b, fmt, byte, d, kv, per, dtype, batch):
    """Infinite where its codes are large: in its 32 columns of the rows that see it (which may be anything there), and nowhere else."""
    n, nq, window, sinks = 100, 5, 40, 2
    if batch > 10 and d == 128:
        batch = 40
    where = [98, 97, 99, 57, 58, 60, 30, 1, 2, 70]        # seen by some queries, by none, by all
    s = Histories(b, [n] * batch, kv, d, fmt, 32, seed=57)
    q = torch.randn(batch, nq, kv * per, d, generator=gen(58)).to(dtype).cuda()
    for i, token in enumerate(where):
        page, at = divmod(int(s.slots[int(s.ends[i]) + token]), 32)
        scales = 32 * (d // 2 if fmt == "mx4" else d) + d // 2
        s.cache.pages[page, i % kv, at // 16, scales + (i % (d // 32)) * 16 + at % 16] = byte
    got = s.cache.attend(q, s.table, s.len_t, window=window, sinks=sinks)
    qn = q.double().cpu().numpy()
    for i in [*range(len(where)), batch - 1]:
        want, off = np.zeros(qn.shape[1:]), np.zeros(qn.shape[1:])
        for h in range(kv * per):
            k, v = (x[s.ends[i]:s.ends[i + 1], h // per] for x in (s.k, s.v))
            want[:, h], off[:, h] = O.attend_rows(qn[i, :, h], k, v, range(n - nq, n), d ** -0.5, window, sinks, dtype)
        result = got[i].clone()
        if i < len(where):
            for x in range(nq):
                if O.sees(n - nq + x, where[i], window, sinks):
                    heads, columns = slice(i % kv * per, (i % kv + 1) * per), slice(i % (d // 32) * 32, (i % (d // 32) + 1) * 32)
                    want[x, heads, columns] = 0.0
                    result[x, heads, columns] = 0.0
        O.assert_close(result, want, off, i)
