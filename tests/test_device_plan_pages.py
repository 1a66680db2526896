"""Free pages of plans made on the device, over many steps: none is lost beside a page table that is wrong."""
import random

import numpy as np
import pytest
import torch

from paper_2502_20727_amd import binding as B
from tests.test_device_plans import BAD_PAGE, RELEASE, Built, check_tables, limits, model
from tests.test_q8_serving import config

gpu_test = pytest.mark.gpu


def step_of(cfg, lim, positions, q_lens, table, free, n_free):
    """The stack's model of a step, beside requests that have an entry that is no page, and a page behind their entries (an earlier step's that refused them): they take
    none, like those whose positions cannot be, and are told so."""
    page, n_pages, rows = cfg.page_size, cfg.n_pages, 0
    at, stuck = list(positions), []
    for b, (p, n) in enumerate(zip(positions, q_lens)):
        rows += n if 0 < n <= lim.q_len else 0
        if 0 < n <= lim.q_len and 0 <= p and p + n <= min(cfg.max_ctx, lim.entries * page) and rows <= lim.tokens:
            there = [0 <= e < n_pages for e in table[b, :-(-(p + n) // page)]]
            held = -(-p // page)
            if not all(there[:held]) and any(there[held:held + 1]):
                at[b] = -1
                stuck.append(b)
    out = model(cfg, lim, at, q_lens, table, free, n_free)
    for b in stuck:
        out["served"][b], out["positions_out"][b] = BAD_PAGE, positions[b]
    return out


def test_the_model_of_a_step_after_a_refused_one():
    cfg, lim = config(page=16, n_pages=10, max_ctx=96), limits(batch=2, tokens=8, q_len=4, entries=6)
    table, free = np.array([[1, 10, -1, -1, -1, -1], [2, -1, -1, -1, -1, -1]], dtype=np.int32), np.array([3, 4, 5, 6, 7, 8, 9, 0, 0, 0], dtype=np.int32)
    one = step_of(cfg, lim, [32, 16], [1, 1], table, free, 7)
    assert one["served"].tolist() == [BAD_PAGE, 1] and one["n_free_out"].tolist() == [5] and one["page_table"][:, 1:3].tolist() == [[10, 9], [8, -1]]
    two = step_of(cfg, lim, [32, 17], [1, 1], one["page_table"], one["free_pages"], 5)
    assert two["served"].tolist() == [BAD_PAGE, 1] and two["n_free_out"].tolist() == [5] and two["positions_out"].tolist() == [32, 18]


class Server:
    """Arrays that steps bring up to date in place, and the model's beside them."""

    def __init__(self, dev, cfg, lim, positions, table, free, n_free):
        self.built, self.cfg, self.lim = Built(dev, cfg, lim, rope=False), cfg, lim
        self.state = list(positions), np.asarray(table, dtype=np.int32), np.asarray(free, dtype=np.int32), n_free
        put = self.built.put
        self.at, self.table, self.free, self.n_free, self.q_lens = put(positions), put(table), put(free), put([n_free]), put([0] * lim.batch)
        self.out = dict(self.built.out, positions_out=self.at, n_free_out=self.n_free)
        self.graph = None

    def launch(self):
        B.spd_pages_build(self.built.dp.ctx, self.built.plan, self.at, self.q_lens, self.table, free_pages=self.free, n_free=self.n_free, **self.out)

    def capture(self):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            self.launch()                       # (nobody has new tokens)
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.launch()

    def step(self, q_lens):
        positions, table, free, n_free = self.state
        want = step_of(self.cfg, self.lim, positions, q_lens, table, free, n_free)
        self.q_lens.copy_(self.built.put(q_lens))
        self.graph.replay() if self.graph else self.launch()
        torch.cuda.synchronize()
        check_tables(self.built, {**self.out, "page_table": self.table, "free_pages": self.free}, want)
        self.state = want["positions_out"].tolist(), want["page_table"], want["free_pages"], int(want["n_free_out"][0])
        return want["served"].tolist()


@gpu_test
@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("q_len,lone", [(1, False), (20, False), (1, True), (2, True)])
def test_no_page_is_lost_beside_a_bad_entry(gpu, graph, q_len, lone):
    """Steps with the same lengths over and over, as a replayed graph makes them, while one request's table holds a page that is none: it takes pages once,
    and the others are served as long as there are pages for them alone."""
    page, steps, bad = 16, 5 if q_len > 2 else 90, 0 if lone else 1
    positions = [48] if lone else [32, 48, 5, 0]
    pages_at = lambda p: -(-p // page)      # noqa: E731
    more = [pages_at(p + (q_len * steps if b != bad else q_len)) - pages_at(p) for b, p in enumerate(positions)]
    kept = [pages_at(p) for p in positions]
    n_pages = sum(kept) + sum(more)
    entries = max(k + m for k, m in zip(kept, more)) + 1
    order, first = [int(p) for p in np.random.RandomState(q_len).permutation(n_pages)], 0
    table = np.full((len(positions), entries), -1, dtype=np.int32)
    for b, k in enumerate(kept):
        table[b, :k] = order[first:first + k]
        first += k
    lost, table[bad, 1] = int(table[bad, 1]), n_pages
    cfg = config(q=8, kv=2, page=page, n_pages=n_pages, max_ctx=entries * page)
    lim = limits(len(positions), q_len * len(positions), q_len, entries)
    server = Server(gpu, cfg, lim, positions, table, order[first:] + [-5] * first, n_pages - first)
    if graph:
        server.capture()
    for i in range(steps):
        assert server.step([q_len] * len(positions)) == [BAD_PAGE if b == bad else q_len for b in range(len(positions))]
        at, table, n_free = server.at.tolist(), server.table.cpu().numpy(), int(server.n_free)
        rows = [table[b, :kept[b] + more[b] if b == bad else pages_at(p)].tolist() for b, p in enumerate(at)]
        there = sum(rows, server.free[:n_free].tolist())
        assert sorted(there + [lost]) == list(range(n_pages + 1))      # every page once, and the entry that is none
    # the entry is mended, and the free list made anew of the pages that are in nobody's positions: the request is served
    assert n_free == 0
    table[bad, 1], free = lost, rows[bad][kept[bad]:]
    server.state = at, table, np.array(free + [-5] * (n_pages - len(free)), dtype=np.int32), len(free)
    server.table.copy_(server.built.put(table))
    server.free.copy_(server.built.put(server.state[2]))
    server.n_free.fill_(len(free))
    assert server.step([q_len if b == bad else 0 for b in range(len(at))]) == [q_len if b == bad else 0 for b in range(len(at))]


@gpu_test
@pytest.mark.parametrize("batch,page", [(7, 16), (64, 32), (300, 16), (1300, 16)])
def test_servers_with_wrong_tables(gpu, batch, page):
    """Requests that come, grow and end, pages that run out, and now and then an entry or a free page that is none: every step as the model has it, pages in rows
    of requests that ended before them among what it finds."""
    r = random.Random(batch)
    entries, n_pages = 8, batch * 4
    cfg = config(q=8, kv=2, d=64, page=page, n_pages=n_pages, max_ctx=entries * page)
    lim = limits(batch, batch * 12, 3 * page, entries)
    server = Server(gpu, cfg, lim, [0] * batch, np.full((batch, entries), -1), np.random.RandomState(batch).permutation(n_pages), n_pages)
    server.capture()
    refused = 0
    for i in range(24):
        positions, table, free, n_free = server.state
        lens = []
        for p in positions:
            kind = r.random()
            lens.append(RELEASE if kind < 0.05 else 0 if kind < 0.1 else r.randint(1, 3 * page) if kind < 0.3 else page if kind < 0.6 else 1)
        for _ in range(max(1, batch // 40) if i % 3 == 1 else 0):
            b = r.randrange(batch)
            held = -(-positions[b] // page)
            if held and r.random() < 0.8:
                table[b, r.randrange(held)] = r.choice([-1, n_pages, 1 << 30])
                server.table.copy_(server.built.put(table))
            elif n_free:
                free[r.randrange(n_free)] = n_pages
                server.free.copy_(server.built.put(free))
        refused += server.step(lens).count(BAD_PAGE)
    assert refused > 0
