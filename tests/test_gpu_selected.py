"""Mean keys of pages, the choice of pages by them, and attention over chosen pages, against 64-bit oracles."""
import numpy as np
import pytest
import torch

import history_oracle as O
from test_gpu_history import BF, HF, F32, Histories, gen, new_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


# ---------------------------------------------------------------------- means
def full_cache(b, pages, page_tokens, kv, d, fmt, seed, scale=1.0):
    c = new_cache(b, pages, page_tokens, kv, d, fmt)
    slots = torch.arange(pages * page_tokens).cuda()
    k = scale * torch.randn(len(slots), kv, d, generator=gen(seed)) * torch.exp(0.5 * torch.randn(d, generator=gen(seed + 1)))
    c.write(k.cuda(), torch.randn(k.shape, generator=gen(seed + 2)).cuda(), slots)
    held = c.read(slots, F32)[0].double().cpu().numpy().reshape(pages, page_tokens, kv, d)
    return c, held


@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("d,kv,page_tokens", [(32, 1, 16), (32, 3, 32), (32, 2, 256), (64, 1, 16), (64, 5, 32), (64, 2, 128), (128, 1, 16), (128, 3, 64), (128, 8, 256)])
def test_means(b, fmt, d, kv, page_tokens):
    """Each of the page's keys added in fp32 (half a step of the sum of magnitudes), a few exchanges, one rounding to bf16."""
    pages = 23
    c, held = full_cache(b, pages, page_tokens, kv, d, fmt, 1)
    which = torch.randperm(pages, generator=gen(4))[:17].int()
    which = torch.cat((which, which[:2], torch.tensor([-1, -1], dtype=torch.int32)))
    means = torch.full((pages, kv, d), 7.0, dtype=BF, device="cuda")
    assert c.summarise(which.cuda(), means) is means
    want, size = held.mean(1), np.abs(held).mean(1)
    named = np.isin(np.arange(pages), which.numpy())
    off = (page_tokens + 8) * 2.0 ** -24 * size + 2.0 ** -8 * np.abs(want) + 2.0 ** -134
    O.assert_close(means[named.tolist()], want[named], off[named])
    assert (means[(~named).tolist()] == 7).all()
    assert c.check()[0] == b.REC_OK
    c.summarise(which[:0].cuda(), means)


def test_means_of_large_and_missing_numbers(b):
    c, held = full_cache(b, 4, 64, 2, 64, "mx4", 5, scale=1e37)
    bad = torch.randn(2, 2, 64, generator=gen(6))
    bad[0, 1, 40] = float("nan")
    c.write(bad.cuda(), bad.cuda(), torch.tensor([70, 71]).cuda())
    held[1, 6:8] = c.read(torch.tensor([70, 71]).cuda(), F32)[0].double().cpu().numpy()
    c.check()
    means = torch.zeros((4, 2, 64), dtype=BF, device="cuda")
    c.summarise(torch.tensor([3, 4, 1, -7, 2 ** 31 - 1], dtype=torch.int32).cuda(), means)
    want = held.mean(1)
    assert np.isnan(want[1, 1, 32:]).all() and not np.isnan(want[1, 0]).any() and np.isfinite(want[3]).all()
    for page in (1, 3):
        O.assert_close(means[page], want[page], 72 * 2.0 ** -24 * np.abs(held[page]).mean(0) + 2.0 ** -8 * np.abs(want[page]))
    assert not means[0].any() and not means[2].any()
    assert c.check() == (b.REC_ERR_INDEX_RANGE, 1, b.REC_FAULT_PAGE)


# --------------------------------------------------------------------- choice
def choice(q, means, table, lengths, page_tokens, count, first, last, candidates):
    """q [B, Q, H, D] and means [pages, kv, D] in float64 -> int [B, Q, kv, count]."""
    nb, nq, heads, _ = q.shape
    kv = means.shape[1]
    per, out = heads // kv, np.full((nb, nq, kv, count), -1)
    for i, n in enumerate(lengths):
        for x in range(nq):
            p = n - 1 if candidates else n - nq + x
            there = p // page_tokens + 1 if p >= 0 else 0
            for h in range(kv):
                rank = []
                for j in range(there):
                    if j < first or j >= there - last:
                        score = np.inf
                        rank.append((-np.inf, -1, j))
                        continue
                    with np.errstate(all="ignore"):
                        s = [float(means[table[i, j], h] @ q[i, x, h * per + y]) for y in range(per)] if 0 <= table[i, j] < len(means) else []
                    s = [y for y in s if not np.isnan(y)]
                    score = max(s) if s else -np.inf
                    rank.append((-score, 0, j))
                chosen = sorted(j for _, _, j in sorted(rank)[:count])
                out[i, x, h, :len(chosen)] = chosen
    return out


def numbers(shape, seed, exact):
    """Normal numbers, or small whole ones whose products tie."""
    x = torch.randn(shape, generator=gen(seed))
    return (x * 1.2).round() if exact else x


class Choices:
    """Tables of histories over a cache whose pages are not looked at."""

    def __init__(self, b, lengths, kv, d, page_tokens, seed, exact=False, spare=3):
        used = [-(-n // page_tokens) for n in lengths]
        total = sum(used) + spare
        order = torch.randperm(total, generator=gen(seed)).tolist()
        self.table = torch.full((len(lengths), max(1, *used)), -1, dtype=torch.int32)
        for i, u in enumerate(used):
            self.table[i, :u] = torch.tensor([order.pop() for _ in range(u)], dtype=torch.int32)
        self.lengths, self.page_tokens = lengths, page_tokens
        self.cache = b.HistoryCache(total, page_tokens, kv, d, "mx4")
        self.means = numbers((total, kv, d), seed + 1, exact).to(BF)
        self.kv, self.d, self.exact = kv, d, exact

    def check(self, q, count, first, last, candidates):
        got = self.cache.select(q.cuda(), self.means.cuda(), self.table.cuda(), torch.tensor(self.lengths, dtype=torch.int32).cuda(), count,
                                first=first, last=last, candidates=candidates)
        four = q[:, None] if q.dim() == 3 else q
        want = choice(four.double().numpy(), self.means.double().numpy(), self.table.numpy(), self.lengths, self.page_tokens, count, first, last, candidates)
        assert got.dtype is torch.int32 and got.shape == (*q.shape[:-2], self.kv, count)
        assert np.array_equal(got.cpu().numpy().reshape(want.shape), want)
        return got


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("d,kv,per,queries,page_tokens,dtype", [(32, 1, 1, 1, 16, BF), (64, 2, 4, 1, 32, HF), (128, 3, 5, 3, 16, BF), (64, 1, 16, 2, 64, HF),
                                                               (32, 2, 17, 2, 32, BF), (128, 1, 40, 1, 16, HF), (64, 4, 2, 20, 16, BF), (32, 3, 1, 40, 16, HF)])
def test_choice(b, exact, d, kv, per, queries, page_tokens, dtype):
    s = Choices(b, [0, 1, page_tokens, page_tokens + 1, 5 * page_tokens, 40 * page_tokens - 3, 17 * page_tokens + 2], kv, d, page_tokens, 21, exact)
    q = numbers((7, queries, kv * per, d), 22, exact).to(dtype)
    for count, first, last in ((1, 0, 1), (4, 1, 1), (7, 3, 4), (6, 0, 2), (33, 2, 1), (64, 1, 1)):
        for candidates in (False, True):
            s.check(q, count, first, last, candidates)
    if queries == 1:
        s.check(q[:, 0], 5, 1, 1, False)
    assert s.cache.check()[0] == b.REC_OK


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("lengths,kv", [([16 * 511, 16 * 513], 2), ([16 * 1500 + 5, 16 * 700], 1), ([16 * 5000, 3], 1), ([16 * 1000, 16 * 600], 2), ([16 * 9000], 1), ([16 * 3000 + 1, 16 * 2500], 2), ([16 * 17000], 1)])
def test_choice_among_many(b, exact, lengths, kv):
    """A row's scores in LDS and in memory, for one wave to sixteen, at once and in several goes."""
    s = Choices(b, lengths, kv, 32, 16, 31, exact)
    q = numbers((len(lengths), 1, kv * 2, 32), 32, exact).to(BF)
    for count, first, last in ((3, 1, 1), (40, 1, 2), (500, 0, 1), (5, 2, 3), (1400, 1, 1)):
        s.check(q, count, first, last, False)


def test_choice_of_equal_scores(b):
    """All alike: the first ones.  Zeros of either sign are one."""
    s = Choices(b, [16 * 900, 16 * 37], 2, 64, 16, 41)
    s.means[:] = 1.0
    q = torch.randn(2, 1, 4, 64, generator=gen(42)).to(BF)
    assert s.check(q, 9, 1, 2, False)[0, 0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 898, 899]
    s.means[::2] = -0.0
    s.means[1::2] = 0.0
    assert s.check(q, 9, 1, 2, False)[0, 0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 898, 899]


def test_choice_by_numbers_that_are_not_finite(b):
    s = Choices(b, [16 * 60, 16 * 9], 1, 32, 16, 51)
    for j, x in ((3, float("nan")), (5, float("inf")), (7, -float("inf")), (9, 3e38), (11, -3e38), (12, 1e-40)):
        s.means[s.table[0, j], 0, 4] = x
    s.means[s.table[0, 20]] = float("nan")
    q = torch.randn(2, 2, 3, 32, generator=gen(52)).to(BF)
    q[0, 1, 2, 4] = 0.0                 # 0 * inf: that product counts for nothing, others do
    q[1, 0, 0, 9] = float("nan")
    q[1, 1, :, 9] = float("inf")
    for count in (4, 12, 57):
        s.check(q, count, 1, 1, True)


def test_choice_reports(b):
    s = Choices(b, [16 * 30, 16 * 50, 16 * 5], 2, 32, 16, 61)
    s.table[1, 8], s.table[1, 12], s.table[2, 1] = len(s.means), -3, 2 ** 31 - 1
    q = torch.randn(3, 1, 2, 32, generator=gen(62)).to(BF)
    s.check(q, 6, 1, 1, False)
    assert s.cache.check() == (b.REC_ERR_INDEX_RANGE, s.table.shape[1] + 8, b.REC_FAULT_PAGE)
    width = s.table.shape[1]
    s.table[s.table < 0] = 0
    s.table[2, 1] = s.table[1, 8] = 0
    lengths = torch.tensor([480, 16 * width + 1, -4], dtype=torch.int32).cuda()
    got = s.cache.select(q.cuda(), s.means.cuda(), s.table.cuda(), lengths, 6)
    s.lengths = [480, 16 * width, 0]
    want = choice(q.double().numpy(), s.means.double().numpy(), s.table.numpy(), s.lengths, 16, 6, 1, 1, False)
    assert np.array_equal(got.cpu().numpy(), want)
    assert s.cache.check() == (b.REC_ERR_LENGTHS, 1, b.REC_FAULT_LENGTH)


# ------------------------------------------------------------------ attention
def expect(s, q, chosen, scale, candidates):
    """Histories s: attention over the chosen pages (numbers, possibly twice)."""
    bq, chosen = q.double().cpu().numpy(), chosen.cpu().numpy()
    nb, nq, heads, d = bq.shape
    out, off, per, page = np.zeros_like(bq), np.zeros_like(bq), heads // s.kv, s.page_tokens
    for i, n in enumerate(s.lengths):
        for x in range(nq):
            p = n - 1 if candidates else n - nq + x
            for h in range(s.kv):
                at = [j for e in chosen[i, x, h] if 0 <= e < s.table.shape[1] for j in range(e * page, e * page + page) if j <= p]
                k, v = (y[s.ends[i]:s.ends[i + 1], h][at] for y in (s.k, s.v))
                rows = slice(h * per, (h + 1) * per)
                out[i, x, rows], off[i, x, rows] = O.attend_rows(bq[i, x, rows], k, v, [len(at) - 1] * per, scale, 0, 0, q.dtype)
    return out, off


def some_pages(s, queries, count, seed):
    """Any pages of the histories' tables, in any order, some twice, some none."""
    g = gen(seed)
    x = torch.randint(-1, s.table.shape[1], (len(s.lengths), queries, s.kv, count), generator=g, dtype=torch.int32)
    return x.cuda()


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("d,kv,per,queries,page_tokens", [(32, 2, 1, 1, 16), (64, 1, 4, 3, 32), (128, 2, 2, 1, 64), (64, 3, 5, 2, 16), (32, 1, 17, 1, 128), (128, 1, 40, 2, 256)])
def test_chosen_pages(b, dtype, fmt, d, kv, per, queries, page_tokens):
    s = Histories(b, [1, 0, 15, 33, page_tokens, 300, 2 * page_tokens + 1, 513], kv, d, fmt, page_tokens)
    q = torch.randn(8, queries, kv * per, d, generator=gen(71)).to(dtype).cuda()
    for count, candidates in ((1, False), (3, False), (3, True), (11, True)):
        chosen = some_pages(s, queries, count, 72 + count)
        got = s.cache.attend_selected(q, chosen, s.table, s.len_t, scale=0.2, candidates=candidates)
        O.assert_close(got, *expect(s, q, chosen, 0.2, candidates), (count, candidates))
    if queries == 1:
        got = s.cache.attend_selected(q[:, 0], chosen[:, 0].contiguous(), s.table, s.len_t)
        O.assert_close(got, *expect(s, q, chosen, d ** -0.5, False))
    assert s.cache.check()[0] == b.REC_OK


@pytest.mark.parametrize("fmt,dtype,d", [("mx4", BF, 64), ("mx8", HF, 128), ("mx8", BF, 32)])
def test_as_attend_where_all_pages_are_chosen(b, fmt, dtype, d):
    s = Histories(b, [700, 1, 0, 64, 65, 1000], 2, d, fmt, 32)
    q = torch.randn(6, 3, 4, d, generator=gen(73)).to(dtype).cuda()
    means = torch.randn(s.cache.pages.shape[0], 2, d, generator=gen(74)).to(BF).cuda()
    for candidates in (False, True):
        chosen = s.cache.select(q, means, s.table, s.len_t, s.table.shape[1], candidates=candidates)
        got = s.cache.attend_selected(q, chosen, s.table, s.len_t, candidates=candidates)
        O.assert_close(got, *s.expect(q, d ** -0.5, 0, 0, candidates))


@pytest.mark.parametrize("batch,count,page_tokens,kv", [(1, 200, 32, 1), (1, 16, 64, 2), (3, 30, 128, 2), (300, 2, 32, 4), (2100, 1, 64, 1), (700, 5, 16, 2), (1200, 9, 16, 4)])
def test_forms_of_a_launch(b, batch, count, page_tokens, kv):
    """Parts in blocks of their own, four waves, two, one; a page's table wider than the choice."""
    n = 256 * page_tokens if batch < 4 else 5 * page_tokens + 3
    s = Histories(b, [n if batch < 4 else 1 + (37 * i) % n for i in range(batch)], kv, 64, "mx4", page_tokens, seed=5)
    q = torch.randn(batch, 1, kv * 2, 64, generator=gen(75)).to(BF).cuda()
    chosen = some_pages(s, 1, count, 76)
    got = s.cache.attend_selected(q, chosen, s.table, s.len_t)
    some = sorted({0, batch - 1, batch // 2, batch // 3})
    s.lengths, ends = [s.lengths[i] for i in some], s.ends
    s.ends = None

    class Some:
        lengths, kv, page_tokens, table = s.lengths, s.kv, s.page_tokens, s.table
    want, off = [], []
    for i, n in zip(some, s.lengths):
        one = Some()
        one.lengths, one.k, one.v, one.ends = [n], s.k[ends[i]:ends[i + 1]], s.v[ends[i]:ends[i + 1]], [0, n]
        x, y = expect(one, q[i:i + 1], chosen[i:i + 1], 64 ** -0.5, False)
        want.append(x[0])
        off.append(y[0])
    O.assert_close(got[some], np.stack(want), np.stack(off))


def test_chosen_pages_that_are_not_there(b):
    """Entries outside the history's table or behind the query, and pages outside the cache: not seen, the first and last reported."""
    s = Histories(b, [200, 130], 2, 64, "mx4", 32, width=9)
    q = torch.randn(2, 1, 4, 64, generator=gen(77)).to(BF).cuda()
    chosen = torch.tensor([[[0, 3, -1], [6, 2, 7]], [[1, 4, 5], [-1, -1, -1]]], dtype=torch.int32).cuda()[:, None].contiguous()
    O.assert_close(s.cache.attend_selected(q, chosen, s.table, s.len_t), *expect(s, q, chosen, 0.125, False))
    assert s.cache.check()[0] == b.REC_OK                    # pages 7 of 6 and 5 of 4 begin behind the query: allowed
    chosen[0, 0, 1, 2], chosen[1, 0, 0, 1] = 9, -2
    got = s.cache.attend_selected(q, chosen, s.table, s.len_t)
    O.assert_close(got, *expect(s, q, chosen, 0.125, False))
    assert s.cache.check() == (b.REC_ERR_INDEX_RANGE, 5, b.REC_FAULT_SLOT)
    chosen[0, 0, 1, 2], chosen[1, 0, 0, 1] = -1, 4
    table = s.table.clone()
    table[1, 1] = len(s.cache.pages)
    got = s.cache.attend_selected(q, chosen, table, s.len_t)
    chosen[1, 0, 0, 0] = -1
    O.assert_close(got, *expect(s, q, chosen, 0.125, False))
    assert s.cache.check() == (b.REC_ERR_INDEX_RANGE, 9 + 1, b.REC_FAULT_PAGE)
    lengths = torch.tensor([-1, 9 * 32 + 5], dtype=torch.int32).cuda()
    assert not s.cache.attend_selected(q, chosen, s.table, lengths)[0].any()
    assert s.cache.check() == (b.REC_ERR_LENGTHS, 0, b.REC_FAULT_LENGTH)


def test_a_number_that_is_not_finite_reaches_only_who_sees_it(b):
    s = Histories(b, [320, 320], 1, 64, "mx8", 32)
    bad = torch.randn(2, 1, 64, generator=gen(78))
    bad[0, 0, 7], bad[1, 0, 50] = float("nan"), float("inf")
    s.cache.write(bad.cuda(), bad.cuda(), s.slots[[5 * 32 + 3, 9 * 32 + 31]].cuda())       # the last token of the first history among them
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    s.cache.check()
    q = torch.randn(2, 3, 2, 64, generator=gen(79)).to(BF).cuda()
    chosen = torch.tensor([[0, 1, 2, 9], [4, 5, 6, 9], [0, 3, 7, 8]], dtype=torch.int32)[None, :, None].expand(2, 3, 1, 4).contiguous().cuda()
    got = s.cache.attend_selected(q, chosen, s.table, s.len_t)
    want, off = expect(s, q, chosen, 0.125, False)
    assert np.isfinite(want[0, [0, 2]]).all() and np.isnan(want[0, 1]).any() and np.isfinite(want[1]).all()
    O.assert_close(got, want, off)
    got = s.cache.attend_selected(q, chosen, s.table, s.len_t, candidates=True)     # the last one is seen by all who chose its page
    want, off = expect(s, q, chosen, 0.125, True)
    assert np.isnan(want[0, 0]).any() and np.isfinite(want[0, 2]).all()
    O.assert_close(got, want, off)


# -------------------------------------------------------------------- together
def test_a_step_over_chosen_pages(b):
    """As a server runs them: events enter, pages that fill up get a mean, queries choose and attend; recorded once, replayed, and
    beside another graph of the same calls on another stream."""
    kv, d, page, users, count = 2, 64, 16, 5, 4
    s = Histories(b, [150, 31, 47, 300, 15], kv, d, "mx4", page, width=24)
    table = s.table.clone()
    free = iter(sorted(set(range(len(s.cache.pages) + 40)) - set(table.flatten().tolist())))
    pages = torch.full((len(s.cache.pages) + 40, *s.cache.pages.shape[1:]), 255, dtype=torch.uint8, device="cuda")
    pages[:len(s.cache.pages)] = s.cache.pages
    cache = b.HistoryCache(len(pages), page, kv, d, "mx4", pages=pages)
    means = torch.zeros(len(pages), kv, d, dtype=BF, device="cuda")
    lengths = s.len_t.clone()
    full = torch.tensor([int(table[u, j]) for u, n in enumerate(s.lengths) for j in range(n // page)], dtype=torch.int32)
    cache.summarise(full.cuda(), means)
    x = torch.zeros(users, 4 + 2 * kv, d, dtype=BF, device="cuda")
    turned = torch.empty(users, 4 + kv, d, dtype=BF, device="cuda")
    slots, filled = torch.zeros(users, dtype=torch.int64, device="cuda"), torch.full((users,), -1, dtype=torch.int32, device="cuda")
    chosen = torch.empty(users, kv, count, dtype=torch.int32, device="cuda")
    out, frequencies = torch.empty(users, 4, d, dtype=BF, device="cuda"), (1e-4 ** (torch.arange(32).double() / 32)).cuda()
    weight = torch.ones(d, device="cuda")

    def step():
        b.rotate_heads(x[:, :4], x[:, 4:4 + kv], lengths, frequencies, weight, weight, q_out=turned[:, :4], k_out=turned[:, 4:])
        cache.write(turned[:, 4:], x[:, 4 + kv:], slots)
        cache.summarise(filled, means)
        cache.select(turned[:, :4], means, table, lengths, count, out=chosen)
        cache.attend_selected(turned[:, :4], chosen, table, lengths, out=out)

    def arrive(seed):
        lengths.add_(1)
        at = lengths.tolist()
        for u, n in enumerate(at):
            if table[u, (n - 1) // page] < 0:
                table[u, (n - 1) // page] = next(free)
        slots.copy_(torch.tensor([int(table[u, (n - 1) // page]) * page + (n - 1) % page for u, n in enumerate(at)]))
        filled.copy_(torch.tensor([int(table[u, (n - 1) // page]) if n % page == 0 else -1 for u, n in enumerate(at)], dtype=torch.int32))
        x.copy_(torch.randn(x.shape, generator=gen(seed)).to(BF))

    arrive(90)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    other, side, theirs = torch.cuda.CUDAGraph(), torch.cuda.Stream(), torch.empty_like(out)
    with torch.cuda.graph(other):
        cache.attend_selected(turned[:, :4], cache.select(turned[:, :4], means, table, lengths, count), table, lengths, out=theirs)
    for i in range(20):
        arrive(91 + i)
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other.replay()
        eager = cache.attend_selected(turned[:, :4], cache.select(turned[:, :4], means, table, lengths, count), table, lengths)
        torch.cuda.synchronize()
        assert torch.equal(eager, out) and torch.equal(theirs, out)
        want = choice(turned[:, None, :4].double().cpu().numpy(), means.double().cpu().numpy(), table.cpu().numpy(), lengths.tolist(), page, count, 1, 1, False)
        assert np.array_equal(chosen.cpu().numpy(), want[:, 0])
        for u, n in enumerate(lengths.tolist()):
            all_slots = torch.tensor([int(table[u, j // page]) * page + j % page for j in range(n)])
            k, v = (y.double().cpu().numpy() for y in cache.read(all_slots.cuda(), F32))
            for h in range(kv):
                rows = slice(2 * h, 2 * h + 2)
                at = [j for e in want[u, 0, h] if e >= 0 for j in range(e * page, min(n, e * page + page))]
                O.assert_close(out[u, rows], *O.attend_rows(turned[u, rows].double().cpu().numpy(), k[at, h], v[at, h], [len(at) - 1] * 2, 0.125, 0, 0, BF), u)
    assert cache.check()[0] == b.REC_OK


def test_strided_queries_and_empty_calls(b):
    s = Histories(b, [100, 40], 2, 64, "mx4", 32)
    rows = torch.randn(2, 5, 9, 64, generator=gen(95)).to(BF).cuda()
    q = rows[:, ::2, 1:9:2]
    means = torch.randn(len(s.cache.pages), 2, 64, generator=gen(96)).to(BF).cuda()
    wide = torch.full((2, 8), -1, dtype=torch.int32, device="cuda")
    wide[:, :s.table.shape[1]] = s.table
    table = wide[:, :s.table.shape[1]]
    chosen = s.cache.select(q, means, table, s.len_t, 2)
    assert torch.equal(chosen, s.cache.select(q.contiguous(), means, s.table, s.len_t, 2))
    got = s.cache.attend_selected(q, chosen, table, s.len_t)
    O.assert_close(got, *expect(s, q.contiguous(), chosen, 0.125, False))
    none = s.cache.select(q[:0], means, table[:0], s.len_t[:0], 2)
    assert none.shape == (0, 3, 2, 2) and s.cache.attend_selected(q[:0], none, table[:0], s.len_t[:0]).shape == (0, 3, 4, 64)
    nothing = s.cache.select(q, means, table[:, :0], torch.zeros_like(s.len_t), 3)
    assert (nothing == -1).all() and not s.cache.attend_selected(q, nothing, table[:, :0], torch.zeros_like(s.len_t)).any()


def test_pages_behind_the_first_4_gib(b):
    """Pages and means at offsets beyond 32 bits: the same calls on the same contents at the start of a small cache."""
    pages, kv, d, page = 2 ** 31 // (8 * 128) + 64, 8, 128, 16
    near, far = (b.HistoryCache(n, page, kv, d, "mx4") for n in (64, pages))
    x = torch.randn(2, 40 * page, kv, d, generator=gen(97))
    at = torch.randperm(40, generator=gen(98))
    lengths = torch.tensor([17 * page + 5, 23 * page - 2], dtype=torch.int32).cuda()
    q = torch.randn(2, 3, 16, d, generator=gen(99)).to(BF).cuda()
    results = []
    for cache, shift in ((near, 24), (far, pages - 40)):
        slots = ((shift + at)[:, None] * page + torch.arange(page)).flatten().cuda()
        cache.write(x[0].cuda(), x[1].cuda(), slots)
        means = torch.empty(len(cache.pages), kv, d, dtype=BF, device="cuda")
        cache.summarise((shift + at).int().cuda(), means)
        table = torch.full((2, 23), -1, dtype=torch.int32)
        table[0, :18], table[1] = (shift + at[:18]).int(), (shift + at[17:]).int()
        table[0, 17] = shift + int(at[39])
        table = table.cuda()
        chosen = cache.select(q, means, table, lengths, 6)
        results.append((means[(shift + at).tolist()], chosen, cache.attend_selected(q, chosen, table, lengths),
                        cache.attend_shared(q, table[0, :7].contiguous(), lengths[:1] - 11 * page, table[:, 7:].contiguous(), lengths - 7 * page)))
        assert cache.check()[0] == b.REC_OK
    for one, other in zip(*results):
        assert torch.equal(one, other)
    assert (results[0][1][:, :, :, 1:5] > 0).all() and results[0][2].isfinite().all() and results[0][3].isfinite().all()


def test_choice_of_many_histories(b):
    """Many histories of as many pages as a wave has keys for, of one more, and of thousands."""
    kv, d, histories, total = 2, 128, 128, 5000
    means = torch.randn(total, kv, d, generator=gen(101)).to(BF).cuda()
    cache = b.HistoryCache(total, 16, kv, d, "mx4")
    for width in (512, 513, 4096):
        table = torch.stack([torch.randperm(total, generator=gen(102 + i))[:width] for i in range(histories)]).int().cuda()
        lengths = torch.randint(8 * width, 16 * width, (histories,), generator=gen(103)).int()
        lengths[0] = 16 * width
        q = torch.randn(histories, 2, d, generator=gen(104)).to(BF).cuda()
        got = cache.select(q, means, table, lengths.cuda(), 9, first=1, last=2)
        scores = torch.stack([means[:, h].double() @ q[:, h].double().t() for h in range(kv)], 1)       # [page, head, history]
        for i, n in enumerate(lengths.tolist()):
            there = -(-n // 16)
            mine = scores[table[i, :there].long(), :, i]
            for h in range(kv):
                best = mine[1:there - 2, h].topk(6).indices + 1
                assert got[i, h].tolist() == [0, *sorted(best.tolist()), there - 2, there - 1]
    assert cache.check()[0] == b.REC_OK
