"""Chosen pages and shared prefixes at the edges of their contract: numbers that are not finite, the range's ends, small weights, nothing outside the buffers."""
import numpy as np
import pytest
import torch

import history_oracle as O
from test_gpu_history import BF, HF, F32, Histories, gen
from test_gpu_history_edges import guarded, poke_value, untouched
from test_gpu_selected import expect, some_pages
from test_gpu_shared_turns import BLOCK_ROWS, Shared

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


def shared_form(b, form, prefix, kv, d, fmt, dtype, page_tokens, seed, rise=0.0):
    """Histories behind a prefix and queries of them whose call has this form."""
    batch, queries = {"joined": (5, 3), "narrow": (63, 5), "wide": (63, BLOCK_ROWS[d, dtype] // 2)}[form]
    s = Shared(b, prefix, [(29 * i + 1) % 150 for i in range(batch)], kv, d, fmt, page_tokens, seed, rise)
    q = s.directed(batch, queries, 4 * kv, dtype, seed + 5)
    assert s.form(q, False)[:2] == (b.REC_OK, dict(joined=b.REC_SHARED_JOINED, narrow=b.REC_SHARED_NARROW, wide=b.REC_SHARED_WIDE)[form])
    return s, q


def with_columns(s, q, got, scale, candidates, columns):
    """s.check() where rows that see a token of the prefix have NaN in `columns` {(kv head, column)} and nowhere else."""
    per, nq = q.shape[2] // s.kv, q.shape[1]
    want = torch.zeros(got.shape, dtype=torch.bool)
    for i, n in enumerate(s.own_lengths):
        for x in range(nq):
            if candidates or n - nq + x >= 0:
                for h, c in columns:
                    want[i, x, h * per:(h + 1) * per, c] = True
    assert torch.equal(got.isnan().cpu(), want), (got.isnan().cpu() != want).nonzero()[:5].tolist()
    s.v = np.nan_to_num(s.v, nan=0.0)
    clean = s.again()               # the same with zeros in their place
    s.check(q, torch.where(want.cuda(), clean, got), scale, candidates)
    assert torch.equal(torch.where(want.cuda(), clean, got), clean)


# ------------------------------------------------------------ values that are not finite
@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
@pytest.mark.parametrize("d,dtype", [(32, BF), (64, HF), (128, BF)])
@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("token", [0, 1277])
def test_a_value_of_the_prefix_that_is_nan(b, form, d, dtype, fmt, token):
    """Its key is finite: its 32 columns are NaN for all who see the prefix, whatever codes are there, others are as with zeros in its place."""
    s, q = shared_form(b, form, 1280 - 2, 2, d, fmt, dtype, 32, seed=token + d)
    slot, block = s.slots[token:token + 1].cuda(), d // 32 - 1
    k = torch.from_numpy(s.k[token:token + 1]).float().cuda()
    v = torch.from_numpy(s.v[token:token + 1]).float().cuda()
    zero = v.clone()
    zero[0, 1, 32 * block:] = 0.0
    bad = zero.clone()
    bad[0, 1, 32 * block + 5] = float("nan")
    for candidates in (False, True):
        s.cache.write(k, bad, slot)
        assert s.cache.check()[0] == b.REC_ERR_VALUE
        got = s.attend(q, scale=0.3, candidates=candidates)
        s.cache.write(k, zero, slot)
        s.v[token, 1, 32 * block:32 * block + 32] = 0.0
        s.again = lambda c=candidates: s.attend(q, scale=0.3, candidates=c)
        with_columns(s, q, got, 0.3, candidates, {(1, 32 * block + j) for j in range(32)})
        assert s.cache.check()[0] == b.REC_OK


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
@pytest.mark.parametrize("d,dtype", [(32, HF), (64, BF), (128, HF)])
def test_codes_of_the_prefix_that_are_nan(b, form, d, dtype):
    """In places that were never written, which a length may count: one column for all who see them, and behind the prefix's end nobody."""
    s, q = shared_form(b, form, 1274, 2, d, "mx8", dtype, 32, seed=21)
    for token, byte in ((3, 0x7f), (640, 0xff), (1273, 0x7f)):
        v = torch.from_numpy(s.v[token:token + 1]).float().cuda()
        v[0, 0, 17] = 0.0
        s.cache.write(torch.from_numpy(s.k[token:token + 1]).float().cuda(), v, s.slots[token:token + 1].cuda())
        s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
        clean = s.attend(q, scale=0.3)
        poke_value(s, token, 0, 17, byte)
        got = s.attend(q, scale=0.3)
        s.again = lambda: clean
        with_columns(s, q, got, 0.3, False, {(0, 17)})
        poke_value(s, token, 0, 17, 0)


@pytest.mark.parametrize("fmt,dtype", [("mx4", BF), ("mx8", HF), ("mx8", BF)])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("batch", [1, 40, 1100])
def test_a_value_that_is_nan_reaches_who_chose_its_page(b, fmt, dtype, d, batch):
    """Its key is finite.  One history in many waves, several, one wave each."""
    s = Histories(b, [700] * batch, 1, d, fmt, 32, seed=31)
    q = torch.randn(batch, 2, 3, d, generator=gen(32)).to(dtype).cuda()
    chosen = torch.stack([torch.randperm(22, generator=gen(33 + i))[:9] for i in range(2 * batch)]).view(batch, 2, 1, 9).int()
    chosen[:, 0, 0, 4], chosen[:, 1][chosen[:, 1] == 7] = 7, 21         # page 7: the first query's, not the second's
    chosen = chosen.cuda()
    clean = s.cache.attend_selected(q, chosen, s.table, s.len_t)
    token, block = 7 * 32 + 19, d // 32 - 1
    at = [int(s.ends[i]) + token for i in range(batch)]
    k, v = (torch.from_numpy(x[at]).float() for x in (s.k, s.v))
    v[:, 0, 32 * block + 1] = float("nan")
    s.cache.write(k.cuda(), v.cuda(), s.slots[at].cuda())
    got = s.cache.attend_selected(q, chosen, s.table, s.len_t)
    want = torch.zeros(got.shape, dtype=torch.bool, device="cuda")
    want[:, 0, :, 32 * block:] = True
    assert torch.equal(got.isnan(), want)
    assert torch.equal(got[:, 1], clean[:, 1]) and torch.equal(got[:, 0, :, :32 * block], clean[:, 0, :, :32 * block])


# --------------------------------------------------- values next to the range's end
@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
@pytest.mark.parametrize("fmt,d", [("mx4", 32), ("mx8", 64), ("mx4", 128), ("mx8", 128)])
def test_means_of_the_largest_values_behind_a_prefix(b, form, fmt, d):
    """A mean of values up to 2^128 is no larger than they are; their sum is."""
    s, q = shared_form(b, form, 1300, 2, d, fmt, BF, 64, seed=41)
    v = torch.sign(torch.randn(1, 2, d, generator=gen(42))) * 2.0 ** 127 * (1 + 0.75 * torch.rand(len(s.slots), 2, d, generator=gen(43)))
    s.cache.write(torch.from_numpy(s.k).float().cuda(), v.cuda(), s.slots.cuda())
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    assert np.abs(s.v).max() > 2.5e38 and np.isfinite(s.v).all()
    s.check(q, s.attend(q, scale=0.3), 0.3, False)


@pytest.mark.parametrize("fmt,d", [("mx4", 32), ("mx8", 64), ("mx4", 128), ("mx8", 128)])
@pytest.mark.parametrize("batch,count", [(1, 90), (3, 40), (1500, 3)])
def test_means_of_the_largest_values_of_chosen_pages(b, fmt, d, batch, count):
    """Parts, several waves, one."""
    s = Histories(b, [32 * max(count, 6) - 5] * batch, 1, d, fmt, 32, seed=51)
    v = torch.sign(torch.randn(1, 1, d, generator=gen(52))) * 2.0 ** 127 * (1 + 0.75 * torch.rand(len(s.slots), 1, d, generator=gen(53)))
    s.cache.write(torch.from_numpy(s.k).float().cuda(), v.cuda(), s.slots.cuda())
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    q = torch.randn(batch, 1, 2, d, generator=gen(54)).to(BF).cuda()
    chosen = some_pages(s, 1, count, 55)
    chosen[..., 0] = 0
    got = s.cache.attend_selected(q, chosen, s.table, s.len_t)
    for i in {0, batch // 2, batch - 1}:
        one = Histories.__new__(Histories)
        one.kv, one.page_tokens, one.table, one.lengths, one.ends = 1, 32, s.table, [s.lengths[i]], [0, s.lengths[i]]
        one.k, one.v = s.k[s.ends[i]:s.ends[i + 1]], s.v[s.ends[i]:s.ends[i + 1]]
        O.assert_close(got[i:i + 1], *expect(one, q[i:i + 1], chosen[i:i + 1], d ** -0.5, False))


# ------------------------------------------------- small weights beside a large one
@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
@pytest.mark.parametrize("d,dtype", [(32, BF), (64, HF), (128, BF), (128, HF)])
@pytest.mark.parametrize("below,at", [(10.0, 650), (17.5, 0), (17.5, 1299)])
def test_many_small_weights_beside_a_large_one(b, form, d, dtype, below, at):
    """One key is e^below more likely than each of the others, and its value is zero, so that the others are the result."""
    s, q = shared_form(b, form, 1300, 2, d, "mx8", dtype, 16, seed=61)
    q = torch.zeros_like(q)
    q[..., 3] = 4.0
    k, v = torch.zeros(len(s.slots), 2, d), torch.rand(len(s.slots), 2, d, generator=gen(62)) + 0.5
    k[at, :, 3], v[at] = below / 4, 0.0
    s.cache.write(k.cuda(), v.cuda(), s.slots.cuda())
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    s.check(q, s.attend(q, scale=1.0), 1.0, False)


# --------------------------------------------------------- nothing outside the buffers
def workspace(need, margin=4096):
    """As many bytes as a call asks for, among others."""
    whole = torch.full((need + 2 * margin,), 0x5A, dtype=torch.uint8, device="cuda")
    return whole, whole[margin:margin + need]


def call_query(b, q, out, table, lengths, scale, candidates):
    return b.rec_query(q.data_ptr(), out, *q.stride()[:3], b._ATTEND_CODES[q.dtype], *q.shape[:3], table.data_ptr(), table.stride(0), table.shape[1],
                       lengths.data_ptr(), scale, 0, 0, int(candidates))


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
@pytest.mark.parametrize("d,dtype", [(32, BF), (32, HF), (64, BF), (64, HF), (128, BF), (128, HF)])
def test_results_and_parts_behind_a_prefix_stay_within_their_buffers(b, form, d, dtype):
    """Rows that end inside a block; a workspace of exactly as many bytes as the call asks for."""
    import ctypes as C
    s, q = shared_form(b, form, 2100, 2, d, "mx4", dtype, 32, seed=71)
    q = q[:-1].contiguous()
    own, lengths = s.own[:-1].contiguous(), s.own_len[:-1].contiguous()
    rows = q.shape[0] * q.shape[1] * q.shape[2]
    buffer, out = guarded(rows, d, dtype)
    query = call_query(b, q, out.data_ptr(), own, lengths, 0.3, False)
    need = b.rec_history_attend_shared_workspace_bytes(s.cache._h, query, len(s.prefix))
    whole, ws = workspace(need)
    st = b._lib.rec_history_attend_shared(C.byref(s.cache._h), C.byref(query), s.prefix.data_ptr(), len(s.prefix), s.prefix_len.data_ptr(),
                                          ws.data_ptr() if need else None, need, b._stream())
    torch.cuda.synchronize()
    assert st == b.REC_OK and untouched(buffer, rows) and bool((whole[:4096] == 0x5A).all()) and bool((whole[4096 + need:] == 0x5A).all())
    s.own_lengths = s.own_lengths[:-1]
    s.check(q, out.view(q.shape), 0.3, False)


@pytest.mark.parametrize("batch,queries,per,count,page_tokens,d,fmt", [(1, 1, 3, 200, 32, 64, "mx4"), (2, 1, 17, 100, 64, 128, "mx8"), (30, 3, 2, 7, 16, 32, "mx8"), (700, 2, 5, 3, 32, 64, "mx4")])
def test_results_and_parts_of_chosen_pages_stay_within_their_buffers(b, batch, queries, per, count, page_tokens, d, fmt):
    import ctypes as C
    lengths = [page_tokens * max(8, count) - 3 * (i % 5) for i in range(batch)]
    s = Histories(b, lengths if batch < 100 else [200 - i % 90 for i in range(batch)], 1, d, fmt, page_tokens, seed=81)
    q = torch.randn(batch, queries, per, d, generator=gen(82)).to(BF).cuda()
    chosen = some_pages(s, queries, count, 83)
    rows = batch * queries * per
    buffer, out = guarded(rows, d, BF)
    query = call_query(b, q, out.data_ptr(), s.table, s.len_t, 0.2, False)
    need = b.rec_history_attend_selected_workspace_bytes(s.cache._h, query, count)
    whole, ws = workspace(need)
    st = b._lib.rec_history_attend_selected(C.byref(s.cache._h), C.byref(query), chosen.data_ptr(), count, ws.data_ptr() if need else None, need, b._stream())
    torch.cuda.synchronize()
    assert st == b.REC_OK and untouched(buffer, rows) and bool((whole[:4096] == 0x5A).all()) and bool((whole[4096 + need:] == 0x5A).all())
    assert torch.equal(out.view(q.shape), s.cache.attend_selected(q, chosen, s.table, s.len_t, scale=0.2))


@pytest.mark.parametrize("batch,queries,per,pages,d", [(3, 1, 2, 40, 64), (2, 5, 5, 300, 128), (2, 3, 4, 700, 32), (1, 1, 1, 5000, 64), (1, 20, 17, 513, 64)])
def test_choices_and_scores_stay_within_their_buffers(b, batch, queries, per, pages, d):
    import ctypes as C
    kv, count = 2, 11
    cache = b.HistoryCache(pages, 16, kv, d, "mx4")
    means = torch.randn(pages, kv, d, generator=gen(91)).to(BF).cuda()
    table = torch.stack([torch.randperm(pages, generator=gen(92 + i)) for i in range(batch)]).int().cuda()
    lengths = torch.tensor([16 * pages - 3 * i for i in range(batch)], dtype=torch.int32).cuda()
    q = torch.randn(batch, queries, kv * per, d, generator=gen(95)).to(HF).cuda()
    n = 4 * batch * queries * kv * count
    buffer, out = workspace(n)
    query = call_query(b, q, None, table, lengths, 1.0, False)
    need = b.rec_history_select_workspace_bytes(cache._h, query, count)
    whole, ws = workspace(need)
    st = b._lib.rec_history_select(C.byref(cache._h), C.byref(query), means.data_ptr(), count, 1, 2, out.data_ptr(), ws.data_ptr() if need else None, need, b._stream())
    torch.cuda.synchronize()
    for x, size in ((buffer, n), (whole, need)):
        assert st == b.REC_OK and bool((x[:4096] == 0x5A).all()) and bool((x[4096 + size:] == 0x5A).all())
    assert torch.equal(out.view(torch.int32).view(batch, queries, kv, count), cache.select(q, means, table, lengths, count, first=1, last=2))


@pytest.mark.parametrize("d,dtype", [(32, F32), (64, BF), (128, HF)])
@pytest.mark.parametrize("tokens,heads,kv", [(1, 1, 1), (37, 5, 2), (1000, 3, 0)])
def test_rotated_rows_stay_within_their_buffers(b, d, dtype, tokens, heads, kv):
    q, k = (torch.randn(tokens, h, d, generator=gen(96 + h)).to(dtype).cuda() for h in (heads, kv))
    at, f = torch.arange(tokens).cuda(), torch.rand(d // 2, generator=gen(99), dtype=torch.float64).cuda()
    (q_buffer, q_out), (k_buffer, k_out) = guarded(tokens * heads, d, dtype), guarded(tokens * kv, d, dtype)
    b.rotate_heads(q, k if kv else None, at, f, q_out=q_out.view(q.shape), k_out=k_out.view(k.shape) if kv else None)
    torch.cuda.synchronize()
    assert untouched(q_buffer, tokens * heads) and untouched(k_buffer, tokens * kv)
    want = b.rotate_heads(q, k if kv else None, at, f)
    assert torch.equal(q_out.view(q.shape), want[0]) and (not kv or torch.equal(k_out.view(k.shape), want[1]))


@pytest.mark.parametrize("d,page_tokens", [(32, 16), (64, 32), (128, 256)])
def test_means_of_named_pages_only(b, d, page_tokens):
    s = Histories(b, [page_tokens * 9], 3, d, "mx8", page_tokens, seed=97)
    pages = len(s.cache.pages)
    buffer, means = guarded(pages * 3, d, BF)
    which = torch.tensor([2, -1, 5, 2], dtype=torch.int32).cuda()
    s.cache.summarise(which, means.view(pages, 3, d))
    torch.cuda.synchronize()
    assert untouched(buffer, pages * 3)
    rest = torch.tensor([i for i in range(pages) if i not in (2, 5)]).cuda()
    assert bool((means.view(torch.uint8).view(pages, -1)[rest] == 0x5A).all())
