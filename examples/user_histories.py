"""Users' histories behind one attention layer, served from the compressed cache.

    python examples/user_histories.py [--users 256] [--candidates 50] [--fmt mx4] [--graph-steps 20]

What a server of a history model does with the calls of include/rec_history.h:

  1. New users: their whole histories (ragged, Poisson(80) events clamped to [1, 200]) attend to
     themselves, and their keys and values enter the cache.
  2. An event per user and step: written, then attended to with everything before it.  The step is
     recorded once and replayed, as lengths, slots and events are device memory.
  3. Ranking: candidates of each user attend to the user's last events and first few.
  4. Some users move to a cache of the other format (as to another tier): read, written.

Weights are random; each stage is checked against plain fp32 attention over what the cache holds.
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2203_07424_amd import binding as rec  # noqa: E402

WIDTH, HEADS, KV_HEADS, DIM, PAGE = 256, 8, 2, 64, 32
WINDOW, SINKS = 150, 4


class Pages:
    """Which page belongs to whom: a list of free ones and, for the kernels, a table of users' pages."""

    def __init__(self, num_pages: int, users: int, most_tokens: int):
        self.free = list(range(num_pages))
        self.of = np.full((users, -(-most_tokens // PAGE)), -1, dtype=np.int32)

    def grow(self, user: int, tokens: int) -> None:
        for i in range(-(-tokens // PAGE)):
            if self.of[user, i] < 0:
                self.of[user, i] = self.free.pop()

    def drop(self, user: int) -> None:
        self.free += [int(p) for p in self.of[user] if p >= 0]
        self.of[user] = -1

    def slots(self, user: int, first: int, last: int) -> np.ndarray:
        at = np.arange(first, last)
        return self.of[user, at // PAGE].astype(np.int64) * PAGE + at % PAGE


def plain(q, k, v, position, window, sinks):
    """q [heads, dim] at `position` over k and v [tokens, kv_heads, dim], fp32."""
    j = torch.arange(len(k), device=q.device)
    seen = (j <= position) & ((position - j < window) | (j < sinks))
    k, v = (x.repeat_interleave(HEADS // KV_HEADS, 1).float() for x in (k, v))
    x = ((k * q.float()).sum(-1) * DIM ** -0.5).masked_fill(~seen[:, None], float("-inf"))     # [tokens, heads]
    return (torch.softmax(x, 0)[..., None] * v).sum(0)


def off_by(got, want) -> float:
    """The largest error, of the largest output.  NaN would pass any bound that is compared with it."""
    if got.shape != want.shape or not (torch.isfinite(got).all() and torch.isfinite(want).all()):
        raise ArithmeticError(f"user_histories: {tuple(got.shape)} against {tuple(want.shape)}, or numbers that are not finite")
    return float((got.float() - want).abs().max() / want.abs().max())


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--users", type=int, default=256)
    ap.add_argument("--candidates", type=int, default=50)
    ap.add_argument("--fmt", choices=["mx4", "mx8"], default="mx4")
    ap.add_argument("--graph-steps", type=int, default=20)
    args = ap.parse_args(argv)

    users, steps = args.users, args.graph_steps
    r = np.random.RandomState(0)
    gen = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda").to(torch.bfloat16)   # noqa: E731
    lengths = np.clip(r.poisson(80, users), 1, 200).astype(np.int32)
    most = int(lengths.max()) + steps + 2
    pages = Pages(users * -(-most // PAGE), users, most)
    cache = rec.HistoryCache(len(pages.free), PAGE, KV_HEADS, DIM, args.fmt)
    project = normal(WIDTH, (HEADS + 2 * KV_HEADS) * DIM) * WIDTH ** -0.5
    worst, times = {}, {}

    def projected(events):
        return (events @ project).view(len(events), HEADS + 2 * KV_HEADS, DIM)

    def rows(x):
        """Queries, keys and values as slices of one product."""
        return x[:, :HEADS], x[:, HEADS:HEADS + KV_HEADS], x[:, HEADS + KV_HEADS:]

    def compare(stage, got, want):
        worst[stage] = max(worst.get(stage, 0.0), off_by(got, want))

    def timed(stage, call):
        torch.cuda.synchronize()
        t = time.perf_counter()
        result = call()
        torch.cuda.synchronize()
        times[stage] = (time.perf_counter() - t) * 1e6
        return result

    some = r.permutation(users)[:8].tolist()

    # 1. Whole new histories.
    q, k, v = rows(projected(normal(int(lengths.sum()), WIDTH)))
    ends = np.cumsum(np.concatenate([[0], lengths]))
    offsets = torch.from_numpy(ends.astype(np.int32)).cuda()
    for u in range(users):
        pages.grow(u, int(lengths[u]))
    slots = torch.from_numpy(np.concatenate([pages.slots(u, 0, int(lengths[u])) for u in range(users)])).cuda()

    def enter():
        out = rec.attend_window(q, k, v, offsets, window=WINDOW, sinks=SINKS, fault=cache.fault)
        cache.write(k, v, slots)
        return out

    enter()
    out = timed("whole histories", enter)
    for u in some:
        a, n = int(ends[u]), int(lengths[u])
        compare("whole histories", out[a + n - 1], plain(q[a + n - 1], k[a:a + n], v[a:a + n], n - 1, WINDOW, SINKS))

    # 2. One event a user and step, recorded once.
    event = torch.zeros(users, HEADS + 2 * KV_HEADS, DIM, dtype=torch.bfloat16, device="cuda")
    query, key, value = rows(event)
    table = torch.empty(pages.of.shape, dtype=torch.int32, device="cuda")
    length, slot = torch.zeros(users, dtype=torch.int32, device="cuda"), torch.zeros(users, dtype=torch.int64, device="cuda")
    answers = torch.empty(users, HEADS, DIM, dtype=torch.bfloat16, device="cuda")

    def step():
        cache.write(key, value, slot)
        cache.attend(query, table, length, window=WINDOW, sinks=SINKS, out=answers)

    def arrive():
        """What comes with a step: places for the new events, and their projection."""
        lengths[:] += 1
        for u in range(users):
            pages.grow(u, int(lengths[u]))
        table.copy_(torch.from_numpy(pages.of))
        length.copy_(torch.from_numpy(lengths))
        slot.copy_(torch.from_numpy(np.concatenate([pages.slots(u, lengths[u] - 1, lengths[u]) for u in range(users)])))
        event.copy_(projected(normal(users, WIDTH)))

    def held(cache, u, n):
        return cache.read(torch.from_numpy(pages.slots(u, 0, n)).cuda(), torch.float32)

    arrive()
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(steps):
        arrive()
        timed("step", graph.replay)
        for u in some[:2]:
            n = int(lengths[u])
            compare("step", answers[u], plain(query[u], *held(cache, u, n), n - 1, WINDOW, SINKS))

    # 3. Candidates.
    q = rows(projected(normal(users * args.candidates, WIDTH)))[0].unflatten(0, (users, args.candidates))
    rank = lambda: cache.attend(q, table, length, window=WINDOW, sinks=SINKS, candidates=True)    # noqa: E731
    rank()
    out = timed("candidates", rank)
    for u in some:
        n, c = int(lengths[u]), u % args.candidates
        compare("candidates", out[u, c], plain(q[u, c], *held(cache, u, n), n - 1, WINDOW, SINKS))

    # 4. A few users to a cache of the other format.
    other = rec.HistoryCache(sum(-(-int(lengths[u]) // PAGE) for u in some), PAGE, KV_HEADS, DIM, "mx8" if args.fmt == "mx4" else "mx4")
    moved = Pages(other.pages.shape[0], len(some), most)
    from_slots = torch.from_numpy(np.concatenate([pages.slots(u, 0, int(lengths[u])) for u in some])).cuda()
    for i, u in enumerate(some):
        moved.grow(i, int(lengths[u]))
        pages.drop(u)
    to_slots = torch.from_numpy(np.concatenate([moved.slots(i, 0, int(lengths[u])) for i, u in enumerate(some)])).cuda()
    timed("move", lambda: other.write(*cache.read(from_slots), to_slots))
    index = torch.tensor(some, device="cuda")
    out = other.attend(q[index], torch.from_numpy(moved.of).cuda(), length[index], window=WINDOW, sinks=SINKS, candidates=True)
    for i, u in enumerate(some):
        n = int(lengths[u])
        k, v = other.read(torch.from_numpy(moved.slots(i, 0, n)).cuda(), torch.float32)
        compare("move", out[i, 0], plain(q[u, 0], k, v, n - 1, WINDOW, SINKS))

    for c in (cache, other):
        status, position, word = c.check()
        if status != rec.REC_OK:
            raise rec.RecError(status, f"user_histories: word {word}, position {position}")
    for stage in worst:
        print(f"{stage:16s} {times[stage]:9.1f} us   off by {worst[stage]:.2g} of the largest output", flush=True)
    return worst


if __name__ == "__main__":
    main()
