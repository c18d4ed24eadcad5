"""Shared prefixes whose parts take several turns of both groups of waves, for every format, type and width: all rows against 64-bit sums."""
import numpy as np
import pytest
import torch

import history_oracle as O
from test_gpu_history import BF, HF, F32, Histories, gen

pytestmark = pytest.mark.gpu
BLOCK_ROWS = {(32, BF): 256, (32, HF): 192, (64, BF): 192, (64, HF): 128, (128, BF): 128, (128, HF): 64}      # of a wide block


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


class Shared(Histories):
    """Histories whose first one is what all others begin with.  rise: how far its scores rise (or fall, for queries the other way) from its
    first token to its last, in units of the exponent, for queries of directed()."""

    def __init__(self, b, prefix, lengths, kv, d, fmt, page_tokens, seed, rise=0.0):
        super().__init__(b, [prefix] + list(lengths), kv, d, fmt, page_tokens, seed)
        used = -(-prefix // page_tokens)
        self.b, self.prefix, self.prefix_len = b, self.table[0, :used].clone(), self.len_t[:1].clone()
        self.own, self.own_len, self.own_lengths = self.table[1:, :max(-(-n // page_tokens) for n in lengths)].contiguous(), self.len_t[1:].clone(), list(lengths)
        self.direction = torch.sign(torch.randn(d, generator=gen(seed + 1)))
        if rise:
            k = 0.3 * torch.randn(prefix, kv, d, generator=gen(seed + 2)) + (rise * torch.arange(prefix)[:, None, None] / prefix) * self.direction
            v = torch.randn(prefix, kv, d, generator=gen(seed + 3))
            self.cache.write(k.cuda(), v.cuda(), self.slots[:prefix].cuda())
            self.k, self.v = (x.double().cpu().numpy() for x in self.cache.read(self.slots.cuda(), F32))

    def directed(self, batch, queries, heads, dtype, seed):
        """Queries of which each goes the keys' way, the other, or neither: <q, direction> is +-1 or near 0."""
        q = 0.3 * torch.randn(batch, queries, heads, self.d, generator=gen(seed))
        ways = torch.randint(-1, 2, (batch, queries, heads, 1), generator=gen(seed + 1))
        return (q + ways * self.direction / self.d).to(dtype).cuda()

    def form(self, q, candidates):
        query = self.b.rec_query(q.data_ptr(), q.data_ptr(), *q.stride()[:3], self.b._ATTEND_CODES[q.dtype], *q.shape[:3], self.own.data_ptr(),
                                 self.own.stride(0), self.own.shape[1], self.own_len.data_ptr(), 1.0, 0, 0, int(candidates))
        return self.b.rec_probe_shared_form(self.cache._h, query, len(self.prefix))

    def attend(self, q, **kw):
        return self.cache.attend_shared(q, self.prefix, self.prefix_len, self.own, self.own_len, **kw)

    def check(self, q, got, scale, candidates, hidden=()):
        """All rows, with the errors that O.attend_rows counts.  hidden: tokens of the prefix that nobody sees."""
        first = [j for j in range(self.ends[1]) if j not in hidden]
        nq, per, u = q.shape[1], q.shape[2] // self.kv, O.EPS[q.dtype]
        for h in range(self.kv):
            k0, v0 = (torch.from_numpy(x[:self.ends[1], h][first]).cuda() for x in (self.k, self.v))
            for i, n in enumerate(self.own_lengths):
                mine = slice(self.ends[1 + i], self.ends[2 + i])
                k, v = (torch.cat((x0, torch.from_numpy(x[mine, h]).cuda())) for x0, x in ((k0, self.k), (v0, self.v)))
                at = torch.full((nq,), n - 1) if candidates else n - nq + torch.arange(nq)
                at = at.cuda().repeat_interleave(per)
                sees = torch.arange(-len(first), n).cuda()[None] <= at[:, None]
                if not candidates:
                    sees &= at[:, None] >= 0
                x = q[i, :, h * per:(h + 1) * per].double().reshape(nq * per, self.d)
                s = (x @ k.t() * scale).masked_fill(~sees, -torch.inf)
                w = torch.nan_to_num(torch.exp(s - s.amax(1, keepdim=True)))
                w /= w.sum(1, keepdim=True).clamp_min(1e-300)
                want = w @ v
                size = abs(scale) * ((x.abs() @ k.abs().t()).masked_fill(~sees, 0).amax(1) * (self.d + 8) * 2.0 ** -24
                                     + 2.0 ** -16 * x.abs().amax(1) * k.abs().sum(1).max())
                off = u * want.abs() + (u + 2 * size[:, None] + 2.0 ** -20) * (w @ v.abs()) + 2.0 ** -25
                g = got[i, :, h * per:(h + 1) * per].double().reshape(nq * per, self.d)
                wrong = ~((g - want).abs() <= off)
                assert not wrong.any(), (i, h, int(wrong.sum()), wrong.nonzero()[:4].tolist(), float(((g - want).abs() / off).max()))
                none = ~sees.any(1)
                assert not g[none].any()


FORMS = [(d, dtype, fmt) for d in (32, 64, 128) for dtype in (BF, HF) for fmt in ("mx4", "mx8")]


def named(form):
    return f"{form[2]}-{form[0]}-{'bf16' if form[1] is BF else 'f16'}"


def wide(s, q, candidates, parts):
    """The form is the one of many rows, and a part has at least six tiles."""
    st, form, splits, _ = s.form(q, candidates)
    tiles = -(-len(s.prefix) * s.page_tokens // 64)
    assert (st, form) == (s.b.REC_OK, s.b.REC_SHARED_WIDE) and (splits > 1) == (parts > 1) and -(-tiles // splits) >= 6, (st, form, splits, tiles)


@pytest.mark.parametrize("form", FORMS, ids=named)
@pytest.mark.parametrize("prefix,page_tokens,rise", [(1216, 32, 0.0), (1217, 64, 8.0), (1331, 16, 30.0), (1280, 256, 120.0)])
def test_many_turns_in_one_part(b, form, prefix, page_tokens, rise):
    """19, 20 and 21 tiles, of which the last is whole, has one token or 51: odd and even turns of the two groups, and rows whose maxima come late,
    early or anywhere."""
    d, dtype, fmt = form
    queries = BLOCK_ROWS[d, dtype] // 2
    s = Shared(b, prefix, [(29 * i + 1) % 150 for i in range(63)], 2, d, fmt, page_tokens, seed=prefix, rise=rise)
    q = s.directed(63, queries, 8, dtype, 3)
    for candidates in (False, True):
        wide(s, q, candidates, 1)
        s.check(q, s.attend(q, scale=1.0, candidates=candidates), 1.0, candidates)
    assert s.cache.check()[0] == b.REC_OK


@pytest.mark.parametrize("form", FORMS, ids=named)
@pytest.mark.parametrize("prefix,rise", [(3970, 0.0), (4030, 60.0)])
def test_many_turns_in_several_parts(b, form, prefix, rise):
    """Parts whose maxima are far apart are joined; the last one is shorter."""
    d, dtype, fmt = form
    s = Shared(b, prefix, [(11 * i) % 60 for i in range(35)], 1, d, fmt, 64, seed=prefix, rise=rise)
    q = s.directed(35, 40, 5, dtype, 5)
    for candidates, scale in ((False, 1.0), (True, -0.7)):
        wide(s, q, candidates, 2)
        s.check(q, s.attend(q, scale=scale, candidates=candidates), scale, candidates)
    assert s.cache.check()[0] == b.REC_OK


@pytest.mark.parametrize("form", FORMS, ids=named)
def test_pages_that_are_not_there_in_later_turns(b, form):
    """Of a prefix of many turns: their tokens are seen by nobody, the first is reported."""
    d, dtype, fmt = form
    queries = BLOCK_ROWS[d, dtype] // 2
    s = Shared(b, 1250, [(29 * i + 1) % 150 for i in range(63)], 2, d, fmt, 16, seed=9, rise=6.0)
    q = s.directed(63, queries, 8, dtype, 7)
    wide(s, q, True, 1)
    bad = [31, 34, 35, 36, 37, 60, 78]
    for i, x in enumerate(bad):
        s.prefix[x] = (len(s.cache.pages), -1, 2 ** 31 - 1, -2 ** 31)[i % 4]
    got = s.attend(q, scale=1.0, candidates=True)
    s.check(q, got, 1.0, True, hidden={16 * x + j for x in bad for j in range(16)})
    assert s.cache.check() == (b.REC_ERR_INDEX_RANGE, 63 * s.own.shape[1] + 31, b.REC_FAULT_PAGE)


@pytest.mark.parametrize("form", FORMS, ids=named)
def test_as_in_narrow_blocks(b, form):
    """The same prefix before few rows, in blocks of 16 with waves that have every fourth tile."""
    d, dtype, fmt = form
    s = Shared(b, 1331, [(29 * i + 1) % 150 for i in range(63)], 2, d, fmt, 32, seed=11, rise=20.0)
    q = s.directed(63, 5, 8, dtype, 13)
    assert s.form(q, False)[:2] == (b.REC_OK, b.REC_SHARED_NARROW)
    for candidates in (False, True):
        s.check(q, s.attend(q, scale=1.0, candidates=candidates), 1.0, candidates)
    assert s.cache.check()[0] == b.REC_OK
