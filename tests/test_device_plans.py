"""Plans of steps made on the device (spd_pages_reserve, spd_pages_build of include/spd_q8.h): refusals on the CPU; on the GPU the tables against a
stack that is worked request by request, and writes and attention against the same step planned on the host, bit by bit."""
import ctypes as C
import math
import random

import numpy as np
import pytest
import torch

from paper_2502_20727_amd import binding as B
from tests.test_q8_serving import LENGTHS, T16, _example, config, rotate, tables

gpu_test = pytest.mark.gpu
RELEASE, BAD_LENGTHS, BAD_PAGE, NO_PAGES = B.SPD_STEP_RELEASE, B.SPD_STEP_LENGTHS, B.SPD_STEP_PAGE, B.SPD_STEP_NO_PAGES
KINDS = [(B.SPD_BF16, B.SPD_E2M1), (B.SPD_F16, B.SPD_E2M1), (B.SPD_BF16, B.SPD_E4M3), (B.SPD_F16, B.SPD_E4M3), (B.SPD_F16, B.SPD_F16)]
KIND_IDS = ["bf16-e2m1", "f16-e2m1", "bf16-e4m3", "f16-e4m3", "f16-f16"]


def limits(batch=4, tokens=64, q_len=32, entries=20, window=0, sinks=0):
    return B.spd_pages_limits(batch, tokens, q_len, entries, window, sinks)


def model(cfg, lim, positions, q_lens, table, free=None, n_free=0):
    """One step, request by request."""
    page, batch, n_pages = cfg.page_size, lim.batch, cfg.n_pages
    most = min(cfg.max_ctx, lim.entries * page)
    table = table.copy()
    stack = None if free is None else list(free[:min(max(n_free, 0), n_pages)])
    rows = [n if 0 < n <= lim.q_len else 0 for n in q_lens]
    begin = [0]
    for n in rows:
        begin.append(begin[-1] + n)
    fine = [positions[b] >= 0 and -1 <= q_lens[b] <= lim.q_len and positions[b] + max(q_lens[b], 0) <= most and begin[b + 1] <= lim.tokens for b in range(batch)]
    held = [-(-p // page) for p in positions]
    out_free = None if free is None else free.copy()
    if stack is not None:
        for b in range(batch):
            if fine[b] and q_lens[b] == RELEASE:
                for i in range(held[b]):
                    if len(stack) < n_pages:
                        out_free[len(stack)] = table[b, i]
                        stack.append(table[b, i])
    served, after = [], []
    row_seq, row_pos, row_slot = (np.full(lim.tokens, -1, dtype=np.int64) for _ in range(3))
    used = 0
    top = 0 if stack is None else len(stack)
    for b in range(batch):
        p, n = positions[b], q_lens[b]
        after.append(p)
        if not fine[b]:
            served.append(BAD_LENGTHS)
            continue
        if n == RELEASE:
            served.append(0)
            after[-1] = 0
            continue
        entries = -(-(p + n) // page) if n else 0
        need = max(0, entries - held[b]) if stack is not None else 0
        if need:
            used += need                        # (those that find none count too: nobody after them is served)
            if used > top:
                served.append(NO_PAGES)
                continue
            for i in range(need):
                table[b, held[b] + i] = stack.pop()
        if any(not 0 <= e < n_pages for e in table[b, :entries]):
            served.append(BAD_PAGE)
            continue
        served.append(n)
        after[-1] = p + n
        for i in range(n):
            row_seq[begin[b] + i], row_pos[begin[b] + i] = b, p + i
            row_slot[begin[b] + i] = int(table[b, (p + i) // page]) * page + (p + i) % page
    return dict(page_table=table, free_pages=out_free, n_free_out=None if stack is None else np.array([len(stack)]), positions_out=np.array(after),
                served=np.array(served), first_row=np.minimum(np.array(begin), lim.tokens), row_seq=row_seq, row_pos=row_pos, row_slot=row_slot)


class Built:
    """A handle, a device plan and the arrays of its steps."""

    def __init__(self, dev, cfg, lim, pool=None, rope=True):
        self.cfg, self.lim, self.dev = cfg, lim, dev
        self.dp = B.DevicePages(cfg, dev, pool=pool, rope=rope)
        self.plan = B.DevicePlan(self.dp, lim)

        def ints(n, t=torch.int32):
            return torch.full((n,), -77, dtype=t, device=dev)
        self.out = dict(n_free_out=ints(1), positions_out=ints(lim.batch), served=ints(lim.batch), first_row=ints(lim.batch + 1), row_seq=ints(lim.tokens),
                        row_pos=ints(lim.tokens), row_slot=ints(lim.tokens, torch.int64))

    def put(self, x):
        return torch.as_tensor(np.asarray(x, dtype=np.int32)).to(self.dev)

    def build(self, positions, q_lens, table, free=None, n_free=None):
        out = dict(self.out)
        self.table = self.put(table)
        if free is None:
            out.pop("n_free_out")
        else:
            out["free_pages"], out["n_free"] = self.put(free), self.put([n_free])
        B.spd_pages_build(self.dp.ctx, self.plan, self.put(positions), self.put(q_lens), self.table, **out)
        return {**out, "page_table": self.table}


def check_tables(built, got, want):
    for name, w in want.items():
        if w is not None:
            assert np.array_equal(got[name].cpu().numpy(), w), name


# ------------------------------------------------------------------------------------------ CPU

@pytest.fixture
def ctx():
    made = []

    def make(**over):
        cfg = config(**over)
        made.append(B.spd_pages_create(cfg))
        return cfg, made[-1]
    yield make
    for c in made:
        B.spd_pages_destroy(c)


@pytest.mark.parametrize("over,code", [
    (dict(batch=0), B.SPD_EINVAL), (dict(tokens=0), B.SPD_EINVAL), (dict(q_len=0), B.SPD_EINVAL), (dict(q_len=65), B.SPD_EINVAL), (dict(entries=0), B.SPD_EINVAL),
    (dict(window=-1), B.SPD_EINVAL), (dict(sinks=3), B.SPD_EINVAL), (dict(window=4, sinks=-1), B.SPD_EINVAL), (dict(batch=4097), B.SPD_EUNSUPPORTED),
    (dict(tokens=(1 << 24) + 1), B.SPD_EUNSUPPORTED), (dict(batch=4096, entries=65537), B.SPD_EUNSUPPORTED), (dict(tokens=1 << 20), B.SPD_EUNSUPPORTED)])
def test_reserve_rejects(ctx, over, code):
    _, pages = ctx()
    with pytest.raises(B.SpdError) as e:
        B.spd_pages_reserve(pages, limits(**over))
    assert e.value.code == code


def test_reserve_sizes(ctx):
    _, pages = ctx()
    n, d = C.c_size_t(), C.c_size_t()
    l = B.lib()
    lim = limits()
    assert l.spd_pages_reserve(None, C.byref(lim), None, 0, C.byref(n), C.byref(d)) == B.SPD_EINVAL
    assert l.spd_pages_reserve(pages, None, None, 0, C.byref(n), C.byref(d)) == B.SPD_EINVAL
    assert l.spd_pages_reserve(pages, C.byref(lim), None, 0, None, C.byref(d)) == B.SPD_EINVAL
    assert l.spd_pages_reserve(pages, C.byref(lim), None, 0, C.byref(n), C.byref(d)) == B.SPD_OK
    buf = np.zeros(n.value, np.uint8)
    assert l.spd_pages_reserve(pages, C.byref(lim), buf.ctypes.data, n.value - 1, C.byref(n), C.byref(d)) == B.SPD_EINVAL
    plan, device = B.spd_pages_reserve(pages, lim)
    info = B.spd_pages_plan_get_info(pages, plan)
    assert info.batch == 4 and info.tokens == 64 and info.held == 0 and device == d.value
    # single tokens need no places for the parts of chunks
    small, _ = B.spd_pages_reserve(pages, limits(q_len=4))
    assert B.spd_pages_plan_get_info(pages, small).workspace_bytes < info.workspace_bytes


def test_calls_refuse_what_they_cannot_work_on(ctx):
    """Host checks alone: nothing is enqueued."""
    cfg, pages = ctx()
    lim = limits()
    plan, device = B.spd_pages_reserve(pages, lim)
    host_made = B.spd_pages_plan(pages, [0], [4], [[1]])
    l, M = B.lib(), 1 << 20
    names = ("positions", "q_lens", "page_table", "free_pages", "n_free", "n_free_out", "positions_out", "served", "first_row", "row_seq", "row_pos", "row_slot")

    def call(pg=pages, ph=plan, pd=64 * M, ld=20, **over):
        at = {n: (i + 1) * M for i, n in enumerate(names)}
        at.update(over)
        s = B.spd_pages_step(at["positions"], at["q_lens"], at["page_table"], ld, *[at[n] for n in names[3:]])
        return l.spd_pages_build(pg, None if ph is None else ph.ctypes.data, pd, C.byref(s), None)
    other = ctx(page=64)[1]
    bad = [dict(pg=None), dict(ph=None), dict(pd=None), dict(pd=64 * M + 8), dict(ph=host_made), dict(pg=other), dict(ld=19), dict(positions=None), dict(q_lens=None),
           dict(page_table=None), dict(free_pages=None), dict(n_free=None), dict(n_free_out=None), dict(positions=M + 2), dict(row_slot=12 * M + 4),
           # memory shared with what is written
           dict(positions_out=M + 4), dict(served=M), dict(served=2 * M), dict(positions_out=2 * M), dict(n_free_out=M), dict(first_row=8 * M - 4), dict(free_pages=3 * M + 4),
           dict(row_seq=3 * M + 20 * 4 * 3), dict(row_pos=10 * M + 255), dict(row_slot=11 * M + 8), dict(n_free=4 * M), dict(n_free_out=4 * M + 8),
           dict(served=64 * M + device - 4), dict(positions=64 * M), dict(page_table=64 * M - 4)]
    for over in bad:
        assert call(**over) == B.SPD_EINVAL, over
    assert l.spd_pages_build(pages, plan.ctypes.data, 64 * M, None, None) == B.SPD_EINVAL
    # a plan made on the device has no lengths that the host knows
    assert l.spd_pages_read(pages, plan.ctypes.data, 64 * M, M, B.SPD_F32, 2 * M, 3 * M, None) == B.SPD_EUNSUPPORTED
    # its limits are those of the matrices
    assert l.spd_pages_attention(pages, plan.ctypes.data, 64 * M, M, 1024, M * 256, M + 63 * 2048, 1024, M * 512, None) == B.SPD_EINVAL


def test_tensors_that_do_not_fit_are_refused(ctx):
    class Plan:
        batch, tokens, entries, n_pages, host_ptr, device_ptr = 4, 64, 20, 40, 0, 0
    B.lib()
    i32 = lambda *n: torch.zeros(*n, dtype=torch.int32)      # noqa: E731
    for args in ((i32(4), i32(4), i32(4, 20)), (i32(4), i32(4), i32(4, 19)), (i32(4), i32(4), i32(80)), (i32(4), i32(4), torch.zeros(4, 20, dtype=torch.int64))):
        with pytest.raises(ValueError):
            B.spd_pages_build(0, Plan, *args)


def test_the_model_itself():
    cfg = config(page=16, n_pages=8)
    got = model(cfg, limits(batch=3, tokens=40, q_len=20, entries=4), [20, 16, 0], [-1, 1, 17], np.array([[5, 6, -1, -1], [2, -1, -1, -1], [-1] * 4]), np.array([7, 0, 0, 0, 0, 0, 0, 0]), 1)
    assert got["n_free_out"].tolist() == [0] and got["page_table"].tolist() == [[5, 6, -1, -1], [2, 6, -1, -1], [5, 7, -1, -1]]
    assert got["positions_out"].tolist() == [0, 17, 17] and got["served"].tolist() == [0, 1, 17] and got["first_row"].tolist() == [0, 0, 1, 18]
    assert got["row_slot"][:3].tolist() == [96, 80, 81] and got["row_slot"][17] == 7 * 16 and got["row_seq"][18] == -1


# ------------------------------------------------------------------------------------------ GPU: tables

def scenario(r, batch, page, n_ctx, chunk, spare, wrong):
    """Lengths, a table and a free list, some of them wrong."""
    positions, q_lens, held = [], [], []
    for _ in range(batch):
        kind = r.random()
        positions.append(r.choice([0, 1, page - 1, page, page + 1, r.randint(0, n_ctx)]))
        q_lens.append(1 if kind < 0.5 else 0 if kind < 0.6 else RELEASE if kind < 0.75 else r.randint(1, chunk))
        held.append(-(-positions[-1] // page))
    entries = -(-(n_ctx + chunk) // page) + 1
    need = sum(max(0, -(-(p + max(n, 0)) // page) - h) for p, n, h in zip(positions, q_lens, held))
    n_pages = sum(held) + max(1, int(need * spare)) + 2
    order = np.random.RandomState(r.randint(0, 1 << 30)).permutation(n_pages)
    table = np.full((batch, entries), -1, dtype=np.int32)
    first = 0
    for b, n in enumerate(held):
        table[b, :n] = order[first:first + n]
        first += n
    free = np.concatenate([order[first:], np.full(first, -5)]).astype(np.int32)
    n_free = n_pages - first
    if wrong:
        for _ in range(max(1, batch // 8)):
            b = r.randrange(batch)
            what = r.randrange(5)
            if what == 0:
                q_lens[b] = r.choice([-2, chunk + 1, 1 << 30, -(1 << 31)])
            elif what == 1:
                positions[b] = r.choice([-1, entries * page, (1 << 31) - 1, -(1 << 31), entries * page + 5])
            elif what == 2 and held[b]:
                table[b, r.randrange(held[b])] = r.choice([-1, n_pages, 1 << 30])
            elif what == 3 and n_free:
                free[r.randrange(n_free)] = r.choice([-1, n_pages])
            else:
                n_free = r.choice([0, n_free // 2])
    return positions, q_lens, table, free, n_free, n_pages, entries


@gpu_test
@pytest.mark.parametrize("batch", [1, 2, 7, 64, 257, 1024, 1025, 2049, 4096])
@pytest.mark.parametrize("wrong", [False, True])
def test_tables_are_those_of_a_stack(gpu, batch, wrong):
    r = random.Random(batch * 2 + wrong)
    for page, n_ctx, chunk, spare, short in ((16, 100, 40, 1.0, 0), (64, 700, 300, 0.6, 0), (16, 33, 2, 1.0, 7), (256, 2000, 5, 1.0, 0)):
        if batch > 1024 and chunk == 300:
            chunk = 20
        positions, q_lens, table, free, n_free, n_pages, entries = scenario(r, batch, page, n_ctx, chunk, spare, wrong)
        tokens = max(chunk, sum(n for n in q_lens if 0 < n <= chunk) + 3 - short)
        cfg = config(q=8, kv=2, d=64, page=page, n_pages=n_pages, cache=B.SPD_E2M1, max_ctx=entries * page)
        lim = limits(batch, tokens, chunk, entries)
        built = Built(gpu, cfg, lim, rope=False)
        check_tables(built, built.build(positions, q_lens, table, free, n_free), model(cfg, lim, positions, q_lens, table, free, n_free))
        # the same without a free list: the table has to be complete
        check_tables(built, built.build(positions, q_lens, table), model(cfg, lim, positions, q_lens, table))


@gpu_test
@pytest.mark.parametrize("page,n_ctx", [(16, 100), (64, 700), (16, 40000), (256, 2000)])
def test_tables_of_a_single_request(gpu, page, n_ctx):
    r = random.Random(n_ctx)
    for i in range(16):
        positions, q_lens, table, free, n_free, n_pages, entries = scenario(r, 1, page, n_ctx, 4, r.choice([1.0, 0.0]), i % 4 == 3)
        tokens = 4 + r.choice([0, 0, 3, 700])
        cfg = config(q=8, kv=2, d=64, page=page, n_pages=n_pages, cache=B.SPD_E2M1, max_ctx=entries * page)
        lim = limits(1, tokens, 4, entries)
        built = Built(gpu, cfg, lim, rope=False)
        check_tables(built, built.build(positions, q_lens, table, free, n_free), model(cfg, lim, positions, q_lens, table, free, n_free))
        check_tables(built, built.build(positions, q_lens, table), model(cfg, lim, positions, q_lens, table))


@gpu_test
def test_a_single_request_in_a_graph(gpu):
    """Grows token by token, ends, and begins anew, by replays of one graph."""
    cfg = config(q=8, kv=2, d=64, page=16, n_pages=12, cache=B.SPD_E2M1, max_ctx=160)
    lim = limits(1, 5, 3, 10)
    built = Built(gpu, cfg, lim, rope=False)
    at, q_lens, n_free, free, table = (built.put(x) for x in ([0], [0], [12], np.arange(12)[::-1], np.full((1, 10), -1)))
    out = dict(built.out, n_free_out=n_free, positions_out=at)

    def step():
        B.spd_pages_build(built.dp.ctx, built.plan, at, q_lens, table, free_pages=free, n_free=n_free, **out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    position, rows, stack, n = [0], np.full((1, 10), -1, dtype=np.int32), free.cpu().numpy(), 12
    r = random.Random(5)
    for _ in range(60):
        lens = [RELEASE if position[0] > 100 and r.random() < 0.2 else r.choice([0, 1, 1, 2, 3, 3, 3])]
        want = model(cfg, lim, position, lens, rows, stack, n)
        q_lens.copy_(built.put(lens))
        graph.replay()
        torch.cuda.synchronize()
        check_tables(built, {**out, "page_table": table, "free_pages": free}, want)
        position, rows, stack, n = want["positions_out"].tolist(), want["page_table"], want["free_pages"], int(want["n_free_out"][0])


@gpu_test
@pytest.mark.parametrize("n_free", [-3, 0, 40, 41, 1 << 30])
def test_counts_of_free_pages_that_cannot_be(gpu, n_free):
    cfg = config(page=16, n_pages=40)
    lim = limits(batch=3, tokens=64, q_len=32, entries=8)
    table = np.array([[1, 2, -1, -1, -1, -1, -1, -1], [3, -1, -1, -1, -1, -1, -1, -1], [4, 5, 6, 7, -1, -1, -1, -1]], dtype=np.int32)
    free = np.arange(40, dtype=np.int32)[::-1].copy()
    built = Built(gpu, cfg, lim)
    args = [32, 10, 60], [20, 8, RELEASE], table, free, n_free
    check_tables(built, built.build(*args), model(cfg, lim, *args))


@gpu_test
def test_long_prompts_of_many_rows(gpu):
    """Chunks beyond the rows that one workgroup writes."""
    cfg = config(q=4, kv=4, d=64, page=16, n_pages=2000, max_ctx=16000)
    lim = limits(batch=3, tokens=12000, q_len=9000, entries=700)
    free = np.random.RandomState(0).permutation(2000).astype(np.int32)
    table = np.full((3, 700), -1, dtype=np.int32)
    table[1, 0] = 1999
    free = np.where(free == 1999, 0, free)
    built = Built(gpu, cfg, lim, rope=False)
    args = [0, 7, 0], [2049, 9000, 1], table, free, 2000
    check_tables(built, built.build(*args), model(cfg, lim, *args))


@gpu_test
def test_outputs_that_are_not_wanted_and_arrays_in_place(gpu):
    cfg = config(page=16, n_pages=40)
    lim = limits(batch=3, tokens=40, q_len=20, entries=6)
    built = Built(gpu, cfg, lim)
    free = np.arange(40, dtype=np.int32)
    table = np.full((3, 6), -1, dtype=np.int32)
    positions, q_lens = [0, 0, 0], [17, 1, 4]
    dev_free, n_free, at, wide = built.put(free), built.put([40]), built.put(positions), built.put(np.concatenate([table, np.full((3, 3), 9)], 1))
    for step in range(4):
        want = model(cfg, lim, positions, q_lens, table, free, int(n_free))
        B.spd_pages_build(built.dp.ctx, built.plan, at, built.put(q_lens), wide, free_pages=dev_free, n_free=n_free, n_free_out=n_free, positions_out=at)
        table, free, positions = want["page_table"], want["free_pages"], want["positions_out"].tolist()
        assert at.tolist() == positions and n_free.tolist() == want["n_free_out"].tolist() and np.array_equal(wide[:, :6].cpu().numpy(), table)
        assert bool((wide[:, 6:] == 9).all()) and np.array_equal(dev_free.cpu().numpy(), free)
        q_lens = [[20, RELEASE, 1], [1, 16, 0], [RELEASE, 1, 5], [1, 1, 1]][step]


# ------------------------------------------------------------------------------------------ GPU: the work, as the host plans it

def both_ways(dev, cfg, positions, q_lens, window=0, sinks=0, spare=5, idle=0, seed=0):
    """The same step planned on both sides: pools, queries and outputs have to be the same bits; rows behind the step stay as they were."""
    ends = [p + n for p, n in zip(positions, q_lens)]
    table = tables(cfg, ends, seed)
    tokens = sum(q_lens)
    width = (cfg.n_q_heads + 2 * cfg.n_kv_heads) * cfg.head_dim
    t = T16[cfg.dtype]
    g = torch.Generator().manual_seed(seed)
    pool = torch.zeros(B.spd_pages_get_sizes(B.spd_pages_create(cfg)).pool_bytes, dtype=torch.uint8, device=dev)
    batch, entries = len(positions) + idle, max([len(x) for x in table] + [1])
    lim = limits(batch, tokens + spare, max(q_lens + [1]), entries, window, sinks)
    built = Built(dev, cfg, lim, pool=pool)
    if sum(positions):
        past = torch.randn(sum(positions), width, generator=g).to(t).to(dev)
        B.spd_pages_write(built.dp.ctx, B.PagePlan(built.dp, [0] * len(positions), positions, table), past, built.dp.rope, pool)
    qkv = torch.randn(tokens + spare, width, generator=g).to(t).to(dev)
    before = pool.clone()
    plan = B.PagePlan(built.dp, positions, q_lens, table, window, sinks)
    q1 = torch.empty(tokens, cfg.n_q_heads * cfg.head_dim, dtype=t, device=dev)
    B.spd_pages_write(built.dp.ctx, plan, qkv[:tokens], built.dp.rope, pool, q1)
    o1 = torch.empty_like(q1)
    B.spd_pages_attention(built.dp.ctx, plan, q1, pool, o1, plan.workspace)
    filled = pool.clone()
    pool.copy_(before)
    full = np.full((batch, entries), -1, dtype=np.int32)
    for b, row in enumerate(table):
        full[b, :len(row)] = row
    built.build(positions + [3] * idle, q_lens + [0] * idle, full)
    q2 = torch.full((tokens + spare, q1.shape[1]), 7.0, dtype=t, device=dev)
    o2 = torch.full_like(q2, 9.0)
    B.spd_pages_write(built.dp.ctx, built.plan, qkv, built.dp.rope, pool, q2)
    B.spd_pages_attention(built.dp.ctx, built.plan, q2, pool, o2, built.plan.workspace)
    assert torch.equal(pool, filled) and torch.equal(q2[:tokens], q1) and torch.equal(o2[:tokens], o1)
    assert bool((q2[tokens:] == 7.0).all()) and bool((o2[tokens:] == 9.0).all())
    return built


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("positions,q_lens", LENGTHS, ids=lambda v: "-".join(map(str, v)))
def test_same_bits_as_planned_on_the_host(gpu, dtype, cache, positions, q_lens):
    both_ways(gpu, config(dtype=dtype, cache=cache, page=32, n_pages=60), list(positions), list(q_lens), idle=2, seed=sum(q_lens))


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("position,q_len", [(0, 1), (15, 1), (16, 2), (1500, 1), (1000, 4)])
def test_same_bits_for_a_single_request(gpu, dtype, cache, position, q_len):
    both_ways(gpu, config(q=8, kv=2, dtype=dtype, cache=cache, page=32, n_pages=60, max_ctx=1600), [position], [q_len], spare=300, seed=position)


@gpu_test
@pytest.mark.parametrize("q,kv,d,page", [(1, 1, 64, 16), (5, 5, 128, 64), (12, 4, 64, 128), (16, 1, 128, 256), (64, 8, 128, 64), (320, 320, 64, 16)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 20)])
def test_same_bits_where_work_is_cut(gpu, q, kv, d, page, window, sinks):
    r = random.Random(q + page)
    few = kv > 100
    for positions, q_lens in (([9000], [1]), ([r.randint(0, 6000) for _ in range(9)], [1] * 9), ([3000, 10, 700], [150, 1, 40]), ([5000], [129]),
                              ([r.randint(0, 900) for _ in range(40)], [1] * 36 + [2, 5, 40, 300])):
        if few:
            positions = [p // 8 for p in positions]
        pages = sum(-(-(p + n) // page) for p, n in zip(positions, q_lens)) + 2
        cfg = config(q=q, kv=kv, d=d, page=page, n_pages=pages, cache=B.SPD_E2M1, max_ctx=9312)
        both_ways(gpu, cfg, positions, q_lens, window, sinks, seed=q)


@gpu_test
@pytest.mark.parametrize("batch", [300, 1500])
def test_same_bits_with_many_requests(gpu, batch):
    r = random.Random(batch)
    positions, q_lens = [r.randint(0, 200) for _ in range(batch)], [r.choice([1, 1, 1, 0, 3]) for _ in range(batch)]
    positions[7], q_lens[11], q_lens[13] = 3000, 100, 60
    pages = sum(-(-(p + n) // 16) for p, n in zip(positions, q_lens)) + 2
    both_ways(gpu, config(q=4, kv=1, d=64, page=16, n_pages=pages, cache=B.SPD_E2M1, max_ctx=4000), positions, q_lens, seed=1)


@gpu_test
@pytest.mark.parametrize("q_len", [1, 40])
def test_requests_that_are_not_served_leave_their_rows(gpu, q_len):
    """Bad lengths, a page outside the pool, no page left: the others are as if alone, their rows where they belong."""
    cfg = config(page=16, n_pages=60, cache=B.SPD_E2M1)
    positions, q_lens = [100, 50, 33, 70, 16], [q_len, q_len, 900, q_len, q_len]
    lim = limits(batch=5, tokens=4 * q_len + 3, q_len=q_len, entries=12)
    built = Built(gpu, cfg, lim)
    width = (cfg.n_q_heads + 2 * cfg.n_kv_heads) * cfg.head_dim
    table = np.full((5, 12), -1, dtype=np.int32)
    order, first = np.random.RandomState(0).permutation(60), 0
    for b, p in enumerate(positions):
        n = -(-p // 16)
        table[b, :n] = order[first:first + n]
        first += n
    past = torch.randn(sum(positions), width, device=gpu).to(torch.bfloat16)
    B.spd_pages_write(built.dp.ctx, B.PagePlan(built.dp, [0] * 5, positions, table), past, built.dp.rope, built.dp.pool)
    table[1, 2] = 60
    need = [-(-(p + q_len) // 16) - -(-p // 16) for p in positions]
    n_free = need[0] + need[1] + need[3]           # nothing is left for the last
    free = np.concatenate([order[first:], np.zeros(first)]).astype(np.int32)
    want = model(cfg, lim, positions, q_lens, table, free, n_free)
    assert want["served"].tolist() == [q_len, BAD_PAGE, BAD_LENGTHS, q_len, NO_PAGES]
    got = built.build(positions, q_lens, table, free, n_free)
    check_tables(built, got, want)
    qkv = torch.randn(lim.tokens, width, device=gpu).to(torch.bfloat16)
    before = built.dp.pool.clone()
    q = torch.full((lim.tokens, 1024), 7.0, dtype=torch.bfloat16, device=gpu)
    out = torch.full_like(q, 9.0)
    B.spd_pages_write(built.dp.ctx, built.plan, qkv, built.dp.rope, built.dp.pool, q)
    B.spd_pages_attention(built.dp.ctx, built.plan, q, built.dp.pool, out, built.plan.workspace)
    pool = built.dp.pool.clone()
    built.dp.pool.copy_(before)
    rows = torch.cat([torch.arange(0, q_len), torch.arange(2 * q_len, 3 * q_len)]).to(gpu)
    there = want["page_table"][[0, 3]]
    plan = B.PagePlan(built.dp, [100, 70], [q_len, q_len], there)
    q1 = torch.empty(2 * q_len, 1024, dtype=torch.bfloat16, device=gpu)
    o1 = torch.empty_like(q1)
    B.spd_pages_write(built.dp.ctx, plan, qkv[rows].contiguous(), built.dp.rope, built.dp.pool, q1)
    B.spd_pages_attention(built.dp.ctx, plan, q1, built.dp.pool, o1, plan.workspace)
    # (the host's plan of the two alone may cut them otherwise: nearly the same where parts are joined, the same bits elsewhere)
    assert torch.equal(pool, built.dp.pool) and torch.equal(q[rows], q1) and torch.allclose(out[rows].float(), o1.float(), rtol=2.0 ** -7, atol=1e-4)
    rest = torch.ones(lim.tokens, dtype=torch.bool, device=gpu)
    rest[rows] = False
    assert bool((q[rest] == 7.0).all()) and bool((out[rest] == 9.0).all())


@gpu_test
@pytest.mark.parametrize("dtype,cache", [KINDS[0], KINDS[2]], ids=[KIND_IDS[0], KIND_IDS[2]])
def test_a_server_in_one_graph(gpu, dtype, cache):
    """Requests come, grow and end; one captured graph of build, write and attention serves every step.  Each step against the host's plan of it, eagerly."""
    cfg = config(dtype=dtype, cache=cache, page=16, n_pages=90, max_ctx=400)
    lim = limits(batch=6, tokens=80, q_len=60, entries=25)
    built = Built(gpu, cfg, lim)
    width, t = (cfg.n_q_heads + 2 * cfg.n_kv_heads) * cfg.head_dim, T16[dtype]
    at, q_lens, n_free = built.put([0] * 6), built.put([0] * 6), built.put([90])
    free, table = built.put(np.random.RandomState(1).permutation(90)), built.put(np.full((6, 25), -1))
    out = dict(built.out, n_free_out=n_free, positions_out=at)
    qkv = torch.zeros(lim.tokens, width, dtype=t, device=gpu)
    q, o = (torch.zeros(lim.tokens, cfg.n_q_heads * cfg.head_dim, dtype=t, device=gpu) for _ in range(2))

    def step():
        B.spd_pages_build(built.dp.ctx, built.plan, at, q_lens, table, free_pages=free, n_free=n_free, **out)
        B.spd_pages_write(built.dp.ctx, built.plan, qkv, built.dp.rope, built.dp.pool, q)
        B.spd_pages_attention(built.dp.ctx, built.plan, q, built.dp.pool, o, built.plan.workspace)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    r = random.Random(3)
    positions, host_table, host_free, host_n = [0] * 6, np.full((6, 25), -1, dtype=np.int32), free.cpu().numpy(), 90
    mirror = torch.zeros_like(built.dp.pool)
    for i in range(24):
        lens = []
        for b in range(6):
            kind = r.random()
            lens.append(RELEASE if positions[b] and kind < 0.1 else 0 if kind < 0.2 else r.randint(1, 40) if positions[b] == 0 and sum(max(x, 0) for x in lens) < 40 else 1)
        lens = [n if n <= 0 or positions[b] + n <= 400 else RELEASE for b, n in enumerate(lens)]
        want = model(cfg, lim, positions, lens, host_table, host_free, host_n)
        fresh = torch.randn(lim.tokens, width, generator=torch.Generator().manual_seed(i)).to(t)
        qkv.copy_(fresh)
        q_lens.copy_(built.put(lens))
        graph.replay()
        torch.cuda.synchronize()
        check_tables(built, {**out, "page_table": table, "free_pages": free}, want)
        assert want["served"].min() >= 0
        live = [b for b in range(6) if lens[b] > 0]
        n = sum(lens[b] for b in live)
        if n:
            # (in the order of the rows; the same requests, so that work is cut the same)
            plan = B.PagePlan(built.dp, [positions[b] for b in live], [lens[b] for b in live], want["page_table"][live])
            q1 = torch.empty(n, q.shape[1], dtype=t, device=gpu)
            o1 = torch.empty_like(q1)
            B.spd_pages_write(built.dp.ctx, plan, qkv[:n], built.dp.rope, mirror, q1)
            B.spd_pages_attention(built.dp.ctx, plan, q1, mirror, o1, plan.workspace)
            assert torch.equal(mirror, built.dp.pool) and torch.equal(q[:n], q1) and torch.equal(o[:n], o1)
        positions, host_table, host_free, host_n = want["positions_out"].tolist(), want["page_table"], want["free_pages"], int(want["n_free_out"][0])


@gpu_test
def test_another_stream_than_the_current_one(gpu):
    cfg = config(page=16, n_pages=60, cache=B.SPD_E2M1)
    built = both_ways(gpu, cfg, [100, 20], [1, 30])
    lim = built.lim
    table = np.full((lim.batch, lim.entries), -1, dtype=np.int32)
    table[:, :lim.entries] = np.arange(lim.batch * lim.entries).reshape(lim.batch, -1)
    want = model(cfg, lim, [100, 20], [1, 30], table)
    pos, lens, dev_table = built.put([100, 20]), built.put([1, 30]), built.put(table)
    out = {k: v for k, v in built.out.items() if k != "n_free_out"}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    B.spd_pages_build(built.dp.ctx, built.plan, pos, lens, dev_table, **out, stream=side)
    side.synchronize()
    check_tables(built, {**out, "page_table": dev_table}, want)


def block_of(ex, cache, max_tokens, n_pages, max_ctx, seed=11):
    from paper_2502_20727_amd import inputs, workloads
    w = workloads.Workload(name="q8-block", hidden=512, n_q_heads=16, n_kv_heads=4, head_dim=64, ffn=1376, n_layers=1, tp=2, dtype=workloads.BF16,
                           seed=seed, batch=3, q_len=1, ctx=64, mask=(1,))
    shard = inputs.layer_shard(w, 0, 1)
    return w, shard, ex.Q8Block(w, shard, 1, max_tokens=max_tokens, n_pages=n_pages, page_size=16, max_ctx=max_ctx, cache=cache)


@gpu_test
@pytest.mark.parametrize("q_len", [1, 12])
@pytest.mark.parametrize("cache", [B.SPD_E2M1, B.SPD_E4M3, B.SPD_BF16], ids=["e2m1", "e4m3", "bf16"])
def test_block_as_one_graph(gpu, cache, q_len):
    """A whole block by a plan made on the device, in one graph, against the block step by step with plans of the host: the same bits, since sums of integers
    are exact, work is cut alike and everything else goes row by row."""
    ex = _example()
    w, _, block = block_of(ex, cache, 40, 60, 300)
    _, _, mirror = block_of(ex, cache, 40, 60, 300)
    batch, rows, g = 5, 20, torch.Generator().manual_seed(7)
    slots = (0.05 * torch.randn(w.tp, rows, w.hidden, generator=g)).to(gpu)
    pool = ex.PagedPool(60, 16)
    steps = ex.GraphSteps(block, pool, [0] * batch, slots, q_len=q_len, window=50, sinks=2)
    r, done = random.Random(q_len), [0] * batch
    for i in range(30):
        lens = [B.SPD_STEP_RELEASE if done[b] > 40 and r.random() < 0.1 else r.randint(0, min(q_len, rows // batch)) for b in range(batch)]
        if q_len > 1 and i % 3 == 0:
            lens = [q_len] + [n if n < 0 else min(n, 2) for n in lens[1:]]
        x = torch.randn(rows, w.hidden, generator=g).to(gpu)
        steps.x.copy_(x)
        steps.q_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out = steps.step()
        assert steps.served.tolist() == [max(n, 0) for n in lens]
        live = [b for b in range(batch) if lens[b] > 0]
        n = sum(lens[b] for b in live)
        if n:
            plan = B.PagePlan(mirror.pages, [done[b] for b in live], [lens[b] for b in live], steps.table[live].cpu().numpy(), window=50, sinks=2)
            peers, again = slots[:, :n].contiguous(), torch.empty(n, w.hidden, device=gpu)
            mirror.forward(plan, x[:n], peers, again)
            assert torch.equal(out[:n], again) and torch.equal(slots[1, :n], peers[1])
            assert torch.equal(block.pages.pool, mirror.pages.pool)
        done = [0 if lens[b] < 0 else done[b] + lens[b] for b in range(batch)]
        assert steps.positions.tolist() == done
        assert int(steps.n_free) == 60 - sum(-(-p // 16) for p in done)
    block.close()
    mirror.close()


@gpu_test
def test_block_over_pages_of_4_bits(gpu):
    """A prompt, then steps as a graph, against the same block in 64 bits with nothing rounded.

    A key or value row of a normal distribution is 11 % off in the root mean square (at most 12 % taken), a row of 8-bit integers 1 %, a product of such rows
    and weights 1.5 %.  An output is a sum of values with probabilities: errors of single values average out as the values themselves do, 12 % of it; an error
    of 12 % of scores of deviation s is one of 12 % s of the probabilities.  Queries, keys, values and the product with O: 1.5 % each.
    In the MLP, gate and up are products of a norm whose error is Y's over X + Y and 1 %, each 1.5 % more, and silu changes by at most 1.1 of its input's change."""
    ex = _example()
    w, shard, block = block_of(ex, B.SPD_E2M1, 200, 60, 300)
    W = {n: torch.from_numpy(a).double() for n, a in shard.items()}
    q, kv, d = w.q_per_rank, w.kv_per_rank, w.head_dim
    pool, g = ex.PagedPool(60, 16), torch.Generator().manual_seed(0)
    past = [[torch.zeros(0, kv, d, dtype=torch.float64) for _ in range(2)] for _ in range(3)]
    done, steps = [0, 0, 0], None

    def norm(t, gain):
        return t / (t.square().mean(-1, keepdim=True) + w.rms_eps).sqrt() * gain

    for lens in ([90, 20, 60], [1, 1, 1], [1, 0, 1], [1, 1, 1]):
        n = sum(lens)
        x = torch.randn(n, w.hidden, generator=g)
        peers = 0.05 * torch.randn(w.tp, n, w.hidden, generator=g)
        if n > 3:
            for s, m in enumerate(lens):
                pool.grow(s, m)
            plan = B.PagePlan(block.pages, done, lens, [pool.table[s] for s in range(3)], window=100, sinks=4)
            slots, out = peers.to(gpu), torch.empty(n, w.hidden, device=gpu)
            block.forward(plan, x.to(gpu), slots, out)
            got = slots[1].cpu().double()
        else:
            if steps is None:
                steps = ex.GraphSteps(block, pool, done, torch.zeros(w.tp, 3, w.hidden, device=gpu), window=100, sinks=4)
            steps.slots[:, :n].copy_(peers)
            steps.x[:n].copy_(x)
            steps.q_lens.copy_(torch.tensor(lens, dtype=torch.int32))
            out = steps.step()[:n]
            got = steps.slots[1, :n].cpu().double()
        X = x.double()
        qkv = norm(X, W["g1"])
        Q, K, V = ((qkv @ W[name]).unflatten(-1, (-1, d)) for name in ("wq", "wk", "wv"))
        att, first, spread = [], 0, []
        for s, m in enumerate(lens):
            at = torch.arange(done[s], done[s] + m)
            mine = slice(first, first + m)
            first += m
            past[s][0] = torch.cat([past[s][0], rotate(K[mine], at, w.rope_base)])
            past[s][1] = torch.cat([past[s][1], V[mine]])
            key = torch.arange(done[s] + m)
            seen = (key <= at[:, None]) & ((key > at[:, None] - 100) | (key < 4))
            qs, o = rotate(Q[mine], at, w.rope_base), torch.zeros(m, q, d, dtype=torch.float64)
            for j in range(q):
                sc = qs[:, j] @ past[s][0][:, j // (q // kv)].t() / math.sqrt(d)
                spread.append(sc[seen])
                o[:, j] = sc.masked_fill(~seen, -math.inf).softmax(-1) @ past[s][1][:, j // (q // kv)]
            att.append(o.flatten(1))
            done[s] += m
        y = torch.cat(att) @ W["wo"]
        m = norm(X + y, W["g2"])
        gate = m @ W["wg"]
        z = (gate * torch.sigmoid(gate) * (m @ W["wu"])) @ W["wd"]
        s2 = float(torch.cat(spread).square().mean())
        of_y = math.sqrt(0.12 ** 2 * (1 + s2) + 4 * 0.015 ** 2)
        of_m = of_y * float(y.norm() / (X + y).norm()) + 0.01
        bound = of_y * float(y.norm()) + (2.1 * (of_m + 0.015) + 0.015) * float(z.norm())
        assert float((got - (y + z)).norm()) < bound
        assert float((out.cpu().double() - (X + peers[0].double() + got)).abs().max()) < 1e-5
    assert steps.positions.tolist() == done
    block.close()


@gpu_test
@pytest.mark.parametrize("cache", [B.SPD_E2M1, B.SPD_E4M3], ids=["e2m1", "e4m3"])
def test_two_plans_on_two_streams(gpu, cache):
    """Sequences of one pool served in two halves, each with a plan, a scratch and a stream of its own, against one stream after the other."""
    cfg = config(page=16, n_pages=400, cache=cache, max_ctx=1200)
    dp = B.DevicePages(cfg, gpu)
    width, cols, t = (cfg.n_q_heads + 2 * cfg.n_kv_heads) * cfg.head_dim, cfg.n_q_heads * cfg.head_dim, T16[cfg.dtype]
    lim, dev = limits(4, 90, 60, 75), gpu
    lens = [[700, 3, 0, 90], [1, 900, 333, 40]], [[1, 60, 5, 1], [1, 1, 1, 50]]
    order = np.random.RandomState(3).permutation(400)
    g = torch.Generator().manual_seed(4)
    halves, first = [], 0
    for h in range(2):
        positions, q_lens = lens[0][h], lens[1][h]
        rows = []
        for p, n in zip(positions, q_lens):
            pages = -(-(p + n) // 16)
            rows.append([int(x) for x in order[first:first + pages]])
            first += pages
        table = np.full((4, 75), -1, dtype=np.int32)
        for b, row in enumerate(rows):
            table[b, :len(row)] = row
        past = torch.randn(sum(positions), width, generator=g).to(t).to(dev)
        B.spd_pages_write(dp.ctx, B.PagePlan(dp, [0] * 4, positions, rows), past, dp.rope, dp.pool)
        put = lambda x: torch.as_tensor(np.asarray(x, dtype=np.int32)).to(dev)      # noqa: E731
        halves.append(dict(plan=B.DevicePlan(dp, lim), at=put(positions), n=put(q_lens), table=put(table), tokens=sum(q_lens),
                           qkv=torch.randn(90, width, generator=g).to(t).to(dev), q=torch.zeros(90, cols, dtype=t, device=dev), o=torch.zeros(90, cols, dtype=t, device=dev)))

    def run(h, stream):
        B.spd_pages_build(dp.ctx, h["plan"], h["at"], h["n"], h["table"], stream=stream)
        B.spd_pages_write(dp.ctx, h["plan"], h["qkv"], dp.rope, dp.pool, h["q"], stream=stream)
        B.spd_pages_attention(dp.ctx, h["plan"], h["q"], dp.pool, h["o"], h["plan"].workspace, stream=stream)
    start = dp.pool.clone()
    for h in halves:
        run(h, None)
    torch.cuda.synchronize()
    want, pool = [h["o"].clone() for h in halves], dp.pool.clone()
    assert all(bool(o[:h["tokens"]].float().abs().sum(1).gt(0).all()) and not bool(o[h["tokens"]:].any()) for o, h in zip(want, halves))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        dp.pool.copy_(start)
        for h in halves:
            h["o"].zero_()
        torch.cuda.synchronize()
        for h, s in zip(halves, streams):
            run(h, s)
        torch.cuda.synchronize()
        assert torch.equal(dp.pool, pool) and all(torch.equal(h["o"], o) for h, o in zip(halves, want))
