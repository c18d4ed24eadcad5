"""Attention of histories that begin with the same tokens, against 64-bit oracles."""
import numpy as np
import pytest
import torch

import history_oracle as O
from test_gpu_history import BF, HF, F32, Histories, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2203_07424_amd import binding
    return binding


@pytest.fixture(autouse=True)
def say(request):
    print(request.node.name, flush=True)


class Shared(Histories):
    """Histories whose first one is what all others begin with.  form: joined if there is little to read, or the prefix's table is so wide that
    few rows take a launch of their own over it, of blocks of 16 rows, or of many."""

    def __init__(self, b, prefix, lengths, kv, d, fmt, page_tokens, seed=0, prefix_width=None, form="joined"):
        super().__init__(b, [prefix] + list(lengths), kv, d, fmt, page_tokens, seed)
        used = -(-prefix // page_tokens)
        tiles = dict(joined=0, narrow=4200 // (len(lengths) * kv) + 1, wide=30001)[form]
        self.prefix = torch.full((max(prefix_width or 1, used, tiles * 64 // page_tokens),), -1, dtype=torch.int32, device="cuda")
        self.prefix[:used] = self.table[0, :used]
        self.prefix_len = torch.tensor([prefix], dtype=torch.int32, device="cuda")
        self.own, self.own_len, self.own_lengths = self.table[1:, :max(1, max([-(-n // page_tokens) for n in lengths]))].contiguous(), self.len_t[1:].clone(), list(lengths)

    def attend(self, q, **kw):
        return self.cache.attend_shared(q, self.prefix, self.prefix_len, self.own, self.own_len, **kw)

    def expect(self, q, scale, candidates, hidden=(), some=None):
        """hidden: tokens of the prefix that nobody sees.  some: only those histories."""
        bq = q.double().cpu().numpy()
        nb, nq, heads, d = bq.shape
        out, off, per = np.zeros_like(bq), np.zeros_like(bq), heads // self.kv
        first = [j for j in range(self.ends[1]) if j not in hidden]
        for i in range(nb) if some is None else some:
            n = self.own_lengths[i]
            for h in range(self.kv):
                mine = slice(self.ends[1 + i], self.ends[2 + i])
                k, v = (np.concatenate((x[:self.ends[1], h][first], x[mine, h])) for x in (self.k, self.v))
                for x in range(nq):
                    p = n - 1 if candidates else n - nq + x
                    if p < 0 and not candidates:
                        continue
                    rows = slice(h * per, (h + 1) * per)
                    out[i, x, rows], off[i, x, rows] = O.attend_rows(bq[i, x, rows], k, v, [len(first) + p] * per, scale, 0, 0, q.dtype)
        return out, off


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
@pytest.mark.parametrize("dtype", [BF, HF], ids=["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["mx4", "mx8"])
@pytest.mark.parametrize("d,kv,per,queries,page_tokens", [(32, 2, 1, 1, 16), (64, 1, 4, 3, 32), (128, 2, 2, 1, 64), (64, 3, 5, 2, 16), (32, 1, 17, 1, 128), (128, 1, 40, 2, 256)])
@pytest.mark.parametrize("prefix", [1, 63, 64, 130, 700])
def test_formula(b, form, dtype, fmt, d, kv, per, queries, page_tokens, prefix):
    """More queries than a history has events leave rows that see nothing; candidates of none see the prefix."""
    s = Shared(b, prefix, [1, 0, 15, 40, 2, 70], kv, d, fmt, page_tokens, seed=prefix, form=form)
    q = torch.randn(6, queries, kv * per, d, generator=gen(81)).to(dtype).cuda()
    for candidates in (False, True):
        got = s.attend(q, scale=0.2, candidates=candidates)
        O.assert_close(got, *s.expect(q, 0.2, candidates), candidates)
    if queries == 1:
        O.assert_close(s.attend(q[:, 0]), *s.expect(q, d ** -0.5, False))
    assert s.cache.check()[0] == b.REC_OK


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
@pytest.mark.parametrize("fmt,dtype,d,kv,per", [("mx4", BF, 64, 1, 2), ("mx8", HF, 128, 2, 1), ("mx8", BF, 32, 2, 4), ("mx4", HF, 64, 1, 1)])
@pytest.mark.parametrize("prefix,batch", [(5000, 1), (5000, 40), (9000, 3), (300, 500), (64, 1300)])
def test_parts(b, form, fmt, dtype, d, kv, per, prefix, batch):
    """Prefixes in many parts, in few, and rows of many histories."""
    s = Shared(b, prefix, [(7 * i) % 41 for i in range(batch)], kv, d, fmt, 32, seed=6, prefix_width=9000 // 32 + 4, form=form)
    q = torch.randn(batch, 1, kv * per, d, generator=gen(82)).to(dtype).cuda()
    some = sorted({0, 1 % batch, batch // 2, batch - 1})
    got = s.attend(q)
    want, off = s.expect(q, d ** -0.5, False, some=some)
    O.assert_close(got[some], want[some], off[some])


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
def test_long_own_parts(b, form):
    """Both the prefix and what comes behind it are divided."""
    s = Shared(b, 4000, [6000], 1, 64, "mx4", 64, form=form)
    q = torch.randn(1, 2, 2, 64, generator=gen(83)).to(BF).cuda()
    O.assert_close(s.attend(q), *s.expect(q, 0.125, False))


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
def test_most_parts(b, form):
    """A row whose long prefix and long history are both divided into as many parts as there may be."""
    s = Shared(b, 20000, [33000], 1, 32, "mx4", 128, form=form)
    q = torch.randn(1, 1, 1, 32, generator=gen(100)).to(BF).cuda()
    O.assert_close(s.attend(q, scale=0.2), *s.expect(q, 0.2, False))


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
def test_nothing_in_front_or_behind(b, form):
    """A prefix of no tokens, of no pages, histories without pages: as attend(), or the prefix alone."""
    s = Shared(b, 0, [5, 0, 90], 2, 64, "mx4", 32, form=form)
    q = torch.randn(3, 2, 4, 64, generator=gen(84)).to(BF).cuda()
    for prefix in (s.prefix, s.prefix[:0]):
        for candidates in (False, True):
            got = s.cache.attend_shared(q, prefix, s.prefix_len, s.own, s.own_len, candidates=candidates)
            O.assert_close(got, *s.expect(q, 0.125, candidates))
    s = Shared(b, 100, [0, 0, 0], 2, 64, "mx4", 32, form=form)
    O.assert_close(s.cache.attend_shared(q, s.prefix, s.prefix_len, s.own[:, :0], s.own_len, candidates=True), *s.expect(q, 0.125, True))
    assert not s.attend(q).any()
    assert s.cache.attend_shared(q[:0], s.prefix, s.prefix_len, s.own[:0], s.own_len[:0]).shape == (0, 2, 4, 64)
    assert s.cache.check()[0] == b.REC_OK


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
def test_numbers_that_are_not_finite(b, form):
    """In the prefix they reach all who see it, in a history's own part its own; behind the prefix's last token nobody."""
    s = Shared(b, 100, [10, 50, 1], 1, 64, "mx8", 32, form=form)          # 28 places of the prefix's last page were never written: NaN
    q = torch.randn(3, 2, 2, 64, generator=gen(85)).to(BF).cuda()
    O.assert_close(s.attend(q), *s.expect(q, 0.125, False))
    bad = torch.randn(1, 1, 64, generator=gen(86))
    bad[0, 0, 40] = float("nan")
    s.cache.write(bad.cuda(), bad.cuda(), s.slots[100 + 3:100 + 4].cuda())      # the first history's fourth event
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    want, off = s.expect(q, 0.125, False)
    assert np.isnan(want[0]).any() and np.isfinite(want[1:]).all()
    O.assert_close(s.attend(q), want, off)
    s.cache.write(bad.cuda(), bad.cuda(), s.slots[98:99].cuda())
    s.k, s.v = (x.double().cpu().numpy() for x in s.cache.read(s.slots.cuda(), F32))
    want, off = s.expect(q, 0.125, False)
    assert np.isnan(want[:2]).any(-1).all() and np.isnan(want[2, 1]).any() and not want[2, 0].any()      # its first query sees nothing
    O.assert_close(s.attend(q), want, off)
    q[1, 0, 0, 3] = float("inf")
    got = s.attend(q)
    assert got[1, 0, 0].isnan().all()


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
def test_reports(b, form):
    s = Shared(b, 200, [40, 33], 2, 64, "mx4", 32, form=form)
    q = torch.randn(2, 1, 4, 64, generator=gen(87)).to(BF).cuda()
    s.prefix[3] = len(s.cache.pages)
    got = s.attend(q)
    O.assert_close(got, *s.expect(q, 0.125, False, hidden=range(96, 128)))
    assert s.cache.check() == (b.REC_ERR_INDEX_RANGE, 2 * s.own.shape[1] + 3, b.REC_FAULT_PAGE)
    s.prefix[3] = -1                    # as attend() has it: no page where the length says that there is one
    O.assert_close(s.attend(q), *s.expect(q, 0.125, False, hidden=range(96, 128)))
    assert s.cache.check() == (b.REC_ERR_INDEX_RANGE, 2 * s.own.shape[1] + 3, b.REC_FAULT_PAGE)
    s.prefix[3] = s.table[0, 3]
    s.prefix_len[0] = 32 * len(s.prefix) + 1
    s.attend(q)
    assert s.cache.check() == (b.REC_ERR_LENGTHS, 2, b.REC_FAULT_LENGTH)
    s.prefix_len[0] = -1
    got = s.attend(q)
    O.assert_close(got, *s.expect(q, 0.125, False, hidden=range(200)))
    assert s.cache.check() == (b.REC_ERR_LENGTHS, 2, b.REC_FAULT_LENGTH)
    s.prefix_len[0], s.own_len[1] = 200, 32 * s.own.shape[1] + 1
    s.attend(q)
    assert s.cache.check() == (b.REC_ERR_LENGTHS, 1, b.REC_FAULT_LENGTH)


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
@pytest.mark.parametrize("scale", [0.0, -0.3])
def test_scales(b, scale, form):
    s = Shared(b, 150, [10, 20], 1, 64, "mx4", 32, form=form)
    q = torch.randn(2, 1, 2, 64, generator=gen(88)).to(BF).cuda()
    O.assert_close(s.attend(q, scale=scale), *s.expect(q, scale, False))


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
def test_strided_queries_and_a_graph(b, form):
    """Events arrive behind the shared tokens; the step is recorded once, beside another graph of the same call on another stream."""
    s = Shared(b, 300, [10, 31, 20], 2, 64, "mx4", 32, form=form)
    rows = torch.randn(3, 9, 64, generator=gen(89)).to(BF).cuda()
    q, out = rows[:, 1:9:2], torch.empty(3, 4, 64, dtype=BF, device="cuda")
    O.assert_close(s.attend(q), *s.expect(q[:, None], 0.125, False))

    def step(out=out):
        return s.attend(q, out=out)

    step()
    torch.cuda.synchronize()
    graph, other, theirs, side = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph(), torch.empty_like(out), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        step()
    with torch.cuda.graph(other):
        step(theirs)
    for i in range(5):
        rows.copy_(torch.randn(3, 9, 64, generator=gen(90 + i)).to(BF))
        s.own_len -= 1
        s.prefix_len -= 13
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            other.replay()
        eager = s.attend(q)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(theirs, eager)
    kept = int(s.prefix_len)
    s.own_lengths = s.own_len.tolist()
    want, off = np.zeros((3, 1, 4, 64)), np.zeros((3, 1, 4, 64))
    ends = s.ends
    for i, n in enumerate(s.own_lengths):
        for h in range(4):
            k, v = (np.concatenate((x[:kept, h // 2], x[ends[1 + i]:ends[1 + i] + n, h // 2])) for x in (s.k, s.v))
            want[i, :, h], off[i, :, h] = O.attend_rows(q[i, h:h + 1].double().cpu().numpy(), k, v, [kept + n - 1], 0.125, 0, 0, BF)
    O.assert_close(out, want, off)


@pytest.mark.parametrize("form", ["joined", "narrow", "wide"])
def test_as_attend_over_the_whole(b, form):
    """A table that begins with the prefix's pages, where the prefix fills them, gives what attend() gives."""
    s = Shared(b, 256, [100, 7, 64], 2, 128, "mx8", 64, form=form)
    q = torch.randn(3, 2, 8, 128, generator=gen(99)).to(HF).cuda()
    whole = torch.cat((s.prefix[:4].expand(3, -1), s.own), 1).contiguous()
    a, z = s.attend(q), s.cache.attend(q, whole, s.own_len + 256)
    want, off = s.expect(q, 128 ** -0.5, False)
    O.assert_close(a, want, off)
    O.assert_close(z, want, off)
