"""Many sequences, many pieces of work and long ones: plans made on the device against the host's, piece by piece and bit by bit; pages in 4 bits
beyond what a wave keeps of them at a time."""
import ctypes as C
import math
import random

import numpy as np
import pytest
import torch

from paper_2502_20727_amd import binding as B
from tests.test_device_plans import Built, both_ways, limits
from tests.test_q4_serving import TYPES, TYPE_IDS, check_attention, config
from tests.test_q8_serving import T16

gpu_test = pytest.mark.gpu


class Header(C.Structure):
    """A plan's first bytes (spd_pages.h)."""
    _fields_ = [("magic", C.c_uint32)] + [(n, C.c_int32) for n in ("batch", "tokens", "window", "sinks", "n_small", "n_large", "n_merge", "n_write")] + \
               [("held", C.c_int64), ("cfg", B.spd_pages_config)] + [(n, C.c_int32) for n in ("seqs", "table", "small", "large", "merge", "write", "merge_rows", "max_end")] + \
               [(n, C.c_size_t) for n in ("bytes", "part_small", "part_large", "workspace")] + \
               [(n, C.c_int32) for n in ("on_device", "q_len", "entries", "reqs", "cuts", "backs", "order")] + [("device_bytes", C.c_size_t)] + \
               [(n, C.c_int32) for n in ("rows", "free0", "top", "n_backs", "sorted")]


SEQ = [("pos", "<i4"), ("q_len", "<i4"), ("tok0", "<i4"), ("table", "<i4"), ("held0", "<i8"), ("end", "<i4"), ("pad", "<i4")]
ITEM = np.dtype(SEQ + [(n, "<i4") for n in ("row0", "sink_blocks", "block0", "first", "count", "slot", "slot0", "parts", "group", "p0", "p1", "p2")])
MERGE = np.dtype(SEQ + [(n, "<i4") for n in ("row0", "rows", "slot0", "parts")])
BLOCK = np.dtype(SEQ + [(n, "<i4") for n in ("block", "p0", "p1", "p2")])


def lists(plan, places=None):
    """The work of a plan (bytes): of few rows, of many, joins, blocks written, each in an order of its own.  `places`: the header that says where they lie."""
    h = Header.from_buffer_copy(plan.tobytes())
    at = h if places is None else places

    def rows(first, n, dtype, fields, whole=()):
        x = np.frombuffer(plan.tobytes(), dtype, n, first)
        out = []
        for r in x:
            row = [int(r[f]) for f in ("pos", "q_len", "tok0", "end") + fields]
            out.append(tuple(row + [int(r[f]) if r["parts"] > 1 else 0 for f in whole]))
        return sorted(out)
    piece = ("row0", "sink_blocks", "block0", "first", "count", "slot", "parts")
    return (rows(at.small, h.n_small, ITEM, piece, ("slot0", "group")), rows(at.large, h.n_large, ITEM, piece, ("slot0",)),
            rows(at.merge, h.n_merge, MERGE, ("row0", "rows", "slot0", "parts")), rows(at.write, h.n_write, BLOCK, ("block",)))


def check_lists(dev, cfg, positions, q_lens, window, sinks):
    """The same pieces, parts, slots, joins and blocks on both sides.  Returns the host's."""
    ends = [p + n for p, n in zip(positions, q_lens)]
    entries, first = -(-max(ends) // cfg.page_size), 0
    table = np.full((len(ends), entries), -1, dtype=np.int32)
    for b, e in enumerate(ends):
        n = -(-e // cfg.page_size)
        table[b, :n] = np.arange(first, first + n)
        first += n
    assert first <= cfg.n_pages
    built = Built(dev, cfg, limits(len(ends), sum(q_lens) + 3, max(q_lens), entries, window, sinks), rope=False)
    want = lists(B.spd_pages_plan(built.dp.ctx, positions, q_lens, table, window, sinks))
    built.build(positions, q_lens, table)
    host = Header.from_buffer_copy(built.plan.host.tobytes())
    got = lists(built.plan.device.cpu().numpy(), host)
    for name, g, w in zip(("few rows", "many rows", "joins", "blocks"), got, want):
        assert g == w, name
    for n, most in zip((len(w) for w in want), (host.n_small, host.n_large, host.n_merge, host.n_write)):
        assert n <= most
    return want


def test_cuts_that_take_as_long_are_told_apart_by_their_order_alone():
    """Of three cuts a plan takes the first that is expected to take the least: in whole numbers, so that host and device agree where two take the same.  (In 64-bit
    floating point the products of such pairs are apart by a rounding, and by another one where they are fused with their sum.)"""
    l = B.lib()
    ties = 0
    for t1 in range(1, 60):
        for s1 in range(2, 257, 3):
            for t2 in range(1, t1 + 1):
                s2, rest = divmod(1650 * t1 + 18 * s1 - 2350 * t2, 18)
                if rest == 0 and 2 <= s2 <= 512:
                    ties += 1
                    assert l.spd_pages_estimate(4 * t1, 256, s1, 1) == l.spd_pages_estimate(4 * t2 - 3, 257, s2, 1) == 1650 * t1 + 3000 + 18 * s1
    assert ties > 1000
    assert l.spd_pages_estimate(9, 200, 0, 3) == 3 * 2 * 2350 and l.spd_pages_estimate(1 << 22, 8704, 512, 1024) == (1 << 20) * 17408 * 2350 + 3000 + 18 * 512 * 1024
    for bad in ((0, 1, 0, 1), (1, 0, 0, 1), (1, 1, -1, 1), (1, 1, 0, 0)):
        assert l.spd_pages_estimate(*bad) == B.SPD_EINVAL


def prompts(r, batch, n_long, q_len, ctx, far, far_ctx):
    """`batch` requests of which `n_long` have chunks, the others single tokens; `far` of either kind, short chunks, lie far behind the rest."""
    q_lens = [r.randint(17, 20) if b < far else r.randint(17, q_len) if b < n_long else r.choice([1, 1, 1, 0, 2]) for b in range(batch)]
    positions = [r.randint(far_ctx // 2, far_ctx) if b < far or batch - b <= far else r.randint(0, ctx) for b in range(batch)]
    order = list(range(batch))
    r.shuffle(order)
    return [positions[b] for b in order], [q_lens[b] for b in order]


@gpu_test
@pytest.mark.parametrize("window,sinks", [(0, 0), (700, 5)])
@pytest.mark.parametrize("q,kv,batch,n_long,q_len,ctx,far,far_ctx", [
    (16, 1, 40, 30, 700, 500, 0, 0), (16, 1, 40, 30, 700, 500, 4, 60000), (16, 1, 130, 125, 900, 300, 2, 200000), (128, 8, 60, 55, 300, 400, 2, 90000),
    (16, 2, 300, 280, 90, 2000, 20, 60000), (16, 1, 1500, 60, 500, 100, 3, 200000), (40, 5, 4096, 900, 30, 60, 3, 50000), (16, 1, 5, 4, 21000, 3000, 1, 300000),
    (16, 16, 200, 0, 20, 2000, 4, 20000)])
def test_pieces_are_the_hosts(gpu, q, kv, batch, n_long, q_len, ctx, far, far_ctx, window, sinks):
    r = random.Random(batch + q_len)
    positions, q_lens = prompts(r, batch, n_long, q_len, ctx, far, far_ctx)
    pages = sum(-(-(p + n) // 64) for p, n in zip(positions, q_lens))
    cfg = config(q=q, kv=kv, d=64, page=64, n_pages=pages, max_ctx=max(positions) + 30000)
    want = check_lists(gpu, cfg, positions, q_lens, window, sinks)
    if far and not window:                      # (fields from behind: few rows parts, slot0, group; many parts, slot0)
        assert any(row[-2] > 1 for row in want[1]) and (not n_long or any(row[-3] > 1 for row in want[0]))


@gpu_test
@pytest.mark.parametrize("kv,blocks", [(2, {2: 15, 57: 3, 368: 7}), (1, {39: 44, 379: 9, 10: 29}), (2, {11: 18, 91: 11, 571: 3}),
                                       (2, {4: 14, 526: 3, 46: 25}), (1, {12: 30, 1284: 1, 197: 21}), (1, {43: 53, 1003: 3, 9: 39})])
def test_cuts_that_are_expected_to_take_as_long(gpu, kv, blocks):
    """Chunks of two tokens behind so many blocks: of the cuts for 256 and 512 workgroups (28 blocks an item, 12) each is expected to take what the other does, and the first
    is taken on both sides."""
    ends = [16 * n for n, times in blocks.items() for _ in range(times)]
    cfg = config(q=16 * kv, kv=kv, d=64, page=64, n_pages=sum(-(-e // 64) for e in ends), max_ctx=max(ends))
    want = check_lists(gpu, cfg, [e - 2 for e in ends], [2] * len(ends), 0, 0)[1]
    longest, items, slots = max(row[8] for row in want), len(want), sum(row[10] > 1 for row in want)
    assert longest == 28 and items * kv <= 256 and B.lib().spd_pages_estimate(longest, items, slots, kv) == B.lib().spd_pages_estimate(12, 512 // kv, slots + 250 // kv, kv)


@gpu_test
def test_pieces_up_to_the_limit(gpu):
    """As many pieces as plans made on the device have room for: 8192."""
    positions, q_lens = [7 * b for b in range(80)], [810 + b % 3 for b in range(80)]
    pieces = sum(-(-n * 16 // 128) for n in q_lens)
    assert 8100 < pieces <= 8192
    cfg = config(q=16, kv=1, d=64, page=16, n_pages=sum(-(-(p + n) // 16) for p, n in zip(positions, q_lens)), max_ctx=2048)
    assert len(check_lists(gpu, cfg, positions, q_lens, 0, 0)[1]) == pieces


@gpu_test
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 20)])
def test_same_bits_of_thousands_of_pieces(gpu, window, sinks):
    r = random.Random(1)
    for q, batch, n_long, q_len, ctx, far in ((16, 40, 36, 600, 200, 2), (16, 1300, 40, 200, 100, 2)):
        positions, q_lens = prompts(r, batch, n_long, q_len, ctx, far, 60000)
        pages = sum(-(-(p + n) // 16) for p, n in zip(positions, q_lens)) + 2
        assert sum(-(-n * q // 128) for n in q_lens if n * q > 16) > (1000 if batch == 40 else 300)
        both_ways(gpu, config(q=q, kv=1, d=64, page=16, n_pages=pages, max_ctx=60100), positions, q_lens, window, sinks, seed=batch)


@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("batch,kv,d,prefix,lone", [(40, 8, 64, 9008, 0), (33, 8, 128, 8336, 0), (2100, 8, 64, 32, 3000), (300, 2, 128, 800, 4000)])
def test_more_sequences_than_workgroups(gpu, dtype, batch, kv, d, prefix, lone):
    """Pages in 4 bits of sequences that are not cut into parts, so that a wave goes through more blocks than it keeps pages of at a time; more of them,
    times heads, than there are counters for parts, one much longer than the rest.  Planned on both sides.  All but that one share their first pages."""
    held_of = -(-(max(prefix, lone) + 16) // 16)
    cfg = config(q=2 * kv, kv=kv, d=d, page=16, n_pages=2 * held_of + batch, dtype=dtype, max_ctx=9100)
    g, t = torch.Generator().manual_seed(batch), T16[dtype]
    common, own = list(range(prefix // 16)), list(range(held_of, 2 * held_of))
    rows = [common + [2 * held_of + b] for b in range(batch)]
    positions = [prefix] * batch
    if lone:
        rows[batch // 2], positions[batch // 2] = own, lone
    entries = max(map(len, rows))
    table = np.full((batch, entries), -1, dtype=np.int32)
    for b, row in enumerate(rows):
        table[b, :len(row)] = row
    built = Built(gpu, cfg, limits(batch, batch + 2, 1, entries))
    dp, width = built.dp, 4 * kv * d
    past = torch.randn(prefix + lone, width, generator=g).to(t).to(gpu)
    B.spd_pages_write(dp.ctx, B.PagePlan(dp, [0, 0], [prefix, lone], [common, own]), past, dp.rope, dp.pool)
    qkv = torch.randn(batch + 2, width, generator=g).to(t).to(gpu)
    before = dp.pool.clone()
    built.build(positions, [1] * batch, table)
    outs = []
    for plan, n in ((built.plan, batch + 2), (B.PagePlan(dp, positions, [1] * batch, table), batch)):
        dp.pool.copy_(before)
        q, out = torch.zeros(n, 2 * kv * d, dtype=t, device=gpu), torch.full((n, 2 * kv * d), math.nan, dtype=t, device=gpu)
        B.spd_pages_write(dp.ctx, plan, qkv[:n], dp.rope, dp.pool, q)
        B.spd_pages_attention(dp.ctx, plan, q, dp.pool, out, plan.workspace)
        outs.append(out[:batch])
        assert not torch.isnan(out[:batch]).any() and bool(torch.isnan(out[batch:]).all())
    assert torch.equal(*outs)
    work = lists(plan.host)[0]
    uncut = max(row[8] for row in work if row[10] == 1)
    assert uncut > 512 if prefix > 8000 else all(row[10] == 1 for row in work) or batch * kv <= 16384
    some = sorted({0, batch // 2, batch - 1, batch // 3})

    class Part:
        window = sinks = 0
    part = Part()
    part.cfg, part.dp, part.positions, part.q_lens, part.table = cfg, dp, [positions[b] for b in some], [1] * len(some), [rows[b] for b in some]
    check_attention(part, outs[0][some], q[some])
