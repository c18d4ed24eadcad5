"""Choices of pages whose scores are in memory: every number of rows of a wave, type and width, ties among them, equal to a 64-bit choice."""
import numpy as np
import pytest
import torch

from test_gpu_history import BF, HF, gen
from test_gpu_selected import numbers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


def choice(q, means, table, lengths, page_tokens, count, first, last, candidates):
    """q [B, Q, H, D], means [pages, kv, D] float64, table of pages that are there -> int [B, Q, kv, count]: highest scores, of equal ones the earlier."""
    nb, nq, heads, _ = q.shape
    kv = means.shape[1]
    per, out = heads // kv, np.full((nb, nq, kv, count), -1)
    for i, n in enumerate(lengths):
        for h in range(kv):
            mine = means[table[i], h]
            for x in range(nq):
                p = n - 1 if candidates else n - nq + x
                there = p // page_tokens + 1 if p >= 0 else 0
                score = (mine[:there] @ q[i, x, h * per:(h + 1) * per].T).max(1)
                score[:first] = score[max(there - last, 0):] = np.inf
                out[i, x, h, :min(there, count)] = np.sort(np.lexsort((np.arange(there), -score))[:count])
    return out


@pytest.mark.parametrize("exact", [False, True], ids=["normal", "ties"])
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("per", [1, 4, 5, 16, 17])
def test_choice_by_scores_in_memory(b, per, d, dtype, exact):
    """More pages than a wave has scores for, and at 128 columns fewer: 300."""
    kv, page_tokens = 2, 16
    for pages in (300, 700, 2500) if d == 128 else (700, 2500):
        lengths = [page_tokens * pages - 3, page_tokens * (pages // 2) + 1, 5]
        total = 2 * pages
        table = np.stack([np.random.RandomState(pages + i).permutation(total)[:pages] for i in range(3)])
        means = numbers((total, kv, d), per + pages, exact).to(BF)
        cache = b.HistoryCache(total, page_tokens, kv, d, "mx4")
        at, n, m = torch.from_numpy(table).int().cuda(), torch.tensor(lengths, dtype=torch.int32).cuda(), means.cuda()
        for queries in (1, 3, 20):
            q = numbers((3, queries, kv * per, d), queries, exact).to(dtype)
            rows = min(queries, max(16 // per, 1)) * min(per, 16)
            for count, first, last in ((9, 1, 2), (64, 0, 1)):
                for candidates in (False, True):
                    query = b.rec_query(16, 16, *q.stride()[:3], b._ATTEND_CODES[dtype], 3, queries, kv * per, at.data_ptr(), pages, pages, n.data_ptr(), 1.0, 0, 0,
                                        int(candidates))
                    st, launches, got_rows, _ = b.rec_probe_select_form(cache._h, query, count)
                    assert (st, got_rows) == (b.REC_OK, rows) and launches == (2 if pages > 512 or rows > 4 else 1)
                    got = cache.select(q.cuda(), m, at, n, count, first=first, last=last, candidates=candidates)
                    want = choice(q.double().numpy(), means.double().numpy(), table, lengths, page_tokens, count, first, last, candidates)
                    assert np.array_equal(got.cpu().numpy(), want), (pages, queries, count, candidates)
        assert cache.check()[0] == b.REC_OK


@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("per,queries", [(4, 3), (17, 2)])
def test_scores_in_memory_that_are_not_finite(b, per, queries, dtype):
    """A product that is NaN counts for nothing; a page outside the cache scores -infinity and is reported."""
    pages, page_tokens, d = 600, 16, 64
    means = numbers((pages, 1, d), 3, True).to(BF)
    means[40, 0, 5], means[41, 0, 5], means[42, 0, 5], means[43] = float("nan"), float("inf"), -float("inf"), float("nan")
    q = numbers((1, queries, per, d), 4, True).to(dtype)
    q[0, -1, 0] = float("nan")
    q[0, 0, -1, 9] = float("inf")
    table = torch.arange(pages, dtype=torch.int32)[None].clone()
    table[0, 17], table[0, 580] = pages, -1
    cache = b.HistoryCache(pages, page_tokens, 1, d, "mx4")
    n = torch.tensor([page_tokens * pages], dtype=torch.int32)
    for count in (5, 300, 597):
        got = cache.select(q.cuda(), means.cuda(), table.cuda(), n.cuda(), count, candidates=True).cpu().numpy()
        for x in range(queries):
            with np.errstate(all="ignore"):
                products = np.stack([(means[:, 0].double().numpy() * q[0, x, y].double().numpy()).sum(1) for y in range(per)])
            products[np.isnan(products)] = -np.inf
            score = products.max(0)
            score[[17, 580]] = -np.inf
            score[[0, -1]] = np.inf
            rank = np.lexsort((np.arange(pages), np.where(np.isin(np.arange(pages), (0, pages - 1)), 0, 1), -score))
            assert got[0, x, 0].tolist() == sorted(rank[:count].tolist()), (count, x)
        assert cache.check() == (b.REC_ERR_INDEX_RANGE, 17, b.REC_FAULT_PAGE)
