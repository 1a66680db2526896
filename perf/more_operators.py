"""Serving over a cache held in 4 bits, steps planned on the GPU, and what is watched of their speed: a paged KV cache whose rows are
brought to 4 bits as they are written and read back, attention of chunks of new tokens (single ones among them) over its pages, and the
building of a step from request lengths that are on the GPU: pages handed out and taken back, the block table, the slot of every new token,
and the work that write and attention are cut into.  Head counts are those of one tensor-parallel rank, or of the whole model, of
paper_2502_20727_amd/workloads.py.

Every operator stands here three times: as a user calls it (`own`), in a plain form of elementary torch operations, and (exact) from its
definition in 64 bits.

A row of the cache goes in groups of 32 features.  A group's scale is 2^e, e the least integer with max|x| <= 7 * 2^e (within the range in
which code * 2^e is a value of the 16-bit type); a code is one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and its sign, the nearest to x * 2^-e, ties
to the even code, 6 for what is beyond.  Keys are rotated in 64 bits, by a rotary table that is given in 32.

A case is a dict; `op` says which operator:
  "attend"   q_heads, kv_heads, head_dim, page, type (queries, output), batch, q_len, ctx (positions before the chunk), ragged (chunks and
             contexts differ), window, sinks, plan ("host" | "device": who planned the step)
  "store"    the same geometry: queries and keys rotated, keys and values quantised into their pages, the pages that hold them read back;
             in: type of the input rows
  "fetch"    the same geometry: everything the sequences hold, back as dense rows of `type`
  "build"    q_heads, kv_heads, head_dim, page, batch (requests), q_len (of a prompt's chunk), ctx, prompts, released (how many of the
             requests have a chunk, and how many hand back their pages; the others have one new token)
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ROPE_BASE = 10000.0
GROUP = 32                                              # features that share a scale
EXPONENTS = {"bf16": (-100, 125), "f16": (-23, 13)}     # of scales, by the pool's 16-bit type


def _pages(name, op, heads, batch, q_len, ctx, type="bf16", page=64, ragged=False, window=0, sinks=0, plan="host", **more):
    q, kv, d = heads
    return {"name": name, "op": op, "q_heads": q, "kv_heads": kv, "head_dim": d, "page": page, "type": type, "batch": batch, "q_len": q_len,
            "ctx": ctx, "ragged": ragged, "window": window, "sinks": sinks, "plan": plan, **more}


def _step(name, heads, batch, ctx, page=64, prompts=0, q_len=1, released=0):
    q, kv, d = heads
    return {"name": name, "op": "build", "q_heads": q, "kv_heads": kv, "head_dim": d, "page": page, "type": "bf16", "batch": batch,
            "q_len": q_len, "ctx": ctx, "prompts": prompts, "released": released}


def listed():
    return [
        # interactive decoding of one sequence on an eighth of the 7B model: latency
        _pages("attend4-7b-step-b1-ctx2048", "attend", (4, 4, 128), 1, 1, 2047),
        # continuous batching on an eighth of the 70B model: 48 sequences of different lengths, one new token each, planned on the GPU
        _pages("attend4-70b-steps-b48-ragged", "attend", (8, 1, 128), 48, 1, 16000, ragged=True, plan="device"),
        # decoding with all heads of the 7B model on one GPU, 16 long sequences: what the cache's bytes are worth
        _pages("attend4-7b-whole-b16-ctx8000", "attend", (32, 32, 128), 16, 1, 8000),
        # chunks of three prompts of a 13B rank behind long contexts, window of 2048 and four sinks, odd lengths, fp16, planned on the GPU
        _pages("attend4-13b-chunks-3x333-window", "attend", (5, 5, 128), 3, 333, 5001, type="f16", page=16, ragged=True, window=2048,
               sinks=4, plan="device"),
        # four prompts of 2048 tokens, all heads of the 70B model on one GPU
        _pages("attend4-70b-prompts-4x2048", "attend", (64, 8, 128), 4, 2048, 0),
        # a decode step of 16 sequences puts away its keys and values
        _pages("store4-70b-steps-b16", "store", (8, 1, 128), 16, 1, 4095, plan="device", **{"in": "bf16"}),
        # four prompts of 2048 tokens do, all heads of the 70B model
        _pages("store4-70b-prompts-4x2048", "store", (64, 8, 128), 4, 2048, 0, **{"in": "bf16"}),
        # sequences handed to another pool or another program: 16 contexts of about 4096 positions read back
        _pages("fetch4-70b-b16-ragged", "fetch", (8, 1, 128), 16, 1, 4095, ragged=True),
        # the same of a 13B rank's 24 contexts of about 8000 in fp16
        _pages("fetch4-13b-b24-ragged", "fetch", (5, 5, 128), 24, 1, 8000, type="f16", page=32, ragged=True),
        # one sequence's next token: latency
        _step("build-b1", (4, 4, 128), 1, 2047),
        # a server's mixed step: 256 requests on an eighth of the 70B model, four of them chunks of prompts, eight that have ended
        _step("build-b256-mixed", (8, 1, 128), 256, 8000, page=16, prompts=4, q_len=512, released=8),
        # a large batch job: 2048 requests, 64 prompts of up to 512 tokens among them, a quarter that ends
        _step("build-b2048-prompts", (8, 1, 128), 2048, 2000, page=32, prompts=64, q_len=512, released=512),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choices(["attend", "store", "fetch", "build"], [6, 2, 2, 3])[0]
    heads = rng.choice([(8, 1, 128), (64, 8, 128), (4, 4, 128), (5, 5, 128), (10, 10, 128), (40, 40, 128), (4, 4, 64), (12, 4, 64), (32, 32, 128)])
    if op == "build":
        heads = rng.choice([(8, 1, 128), (64, 8, 128), (4, 4, 128), (5, 5, 128), (12, 4, 64)])
        batch = _log_int(rng, 1, 2048)
        prompts = rng.choice([0, rng.randint(0, min(batch, 64))])
        c = _step("", heads, batch, _log_int(rng, 16, min(32000, 8_000_000 // batch)), page=rng.choice([16, 32, 64, 128]), prompts=prompts,
                  q_len=_log_int(rng, 2, 512) if prompts else 1, released=rng.choice([0, rng.randint(0, batch - prompts)]))
    else:
        step = rng.random() < (0.6 if op != "fetch" else 1.0)
        batch = _log_int(rng, 1, 64) if step else _log_int(rng, 1, 6)
        q_len = rng.choice([1, 1, 1, rng.randrange(2, 6)]) if step else _log_int(rng, 16, 3000)
        room = min(32000, 4_000_000 // (batch * heads[1]))
        ctx = _log_int(rng, 16, max(32, room)) if step else rng.choice([0, _log_int(rng, 16, 8000)])
        pairs = (1 << 30) // (batch * heads[0])           # the plain form keeps every score: queries x keys of a head
        while q_len > 1 and q_len * (ctx + q_len) > pairs:
            q_len, ctx = (q_len + 1) // 2, ctx // 2
        type = rng.choice(["bf16", "bf16", "f16"])
        more = {"in": rng.choice([type, "f32"])} if op == "store" else {}
        window = rng.choice([0, 0, _log_int(rng, 16, 4096)]) if op == "attend" else 0
        c = _pages("", op, heads, batch, q_len, ctx, type=type, page=rng.choice([16, 32, 64, 128]), ragged=rng.random() < 0.6, window=window,
                   sinks=rng.choice([0, 4, rng.randrange(1, 100)]) if window else 0,
                   plan=rng.choice(["host", "device"]) if op != "fetch" else "host", **more)
    c.pop("name", None)
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed, key):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + key * 7919) % (2 ** 62))
    return g


def _randn(seed, key, *shape):
    return torch.randn(*shape, generator=_generator(seed, key), device="cuda")


def _lengths(case):
    """(positions before the chunk, new tokens) of each sequence: part of the case, whatever the seed."""
    b, n, ctx = case["batch"], case["q_len"], case["ctx"]
    r = random.Random(b * 1000003 + n * 7919 + ctx)
    if case["op"] == "build":
        kinds = [n] * case["prompts"] + [-1] * case["released"] + [1] * (b - case["prompts"] - case["released"])
        r.shuffle(kinds)
        return ([r.randint(ctx // 4, ctx) if k != n or n == 1 else r.choice([0, r.randint(0, ctx)]) for k in kinds],
                [r.randint(max(1, n // 2), n) if k == n else k for k in kinds])
    if not case["ragged"]:
        return [ctx] * b, [n] * b
    return ([ctx] + [r.randint(ctx // 4, ctx) for _ in range(b - 1)], [n] + [r.randint(max(1, n // 2), n) for _ in range(b - 1)])


class _State:
    pass


def _sections(case):
    """Bytes of one head's share of a page: codes of its keys, of its values, scales of its keys, of its values."""
    p, d = case["page"], case["head_dim"]
    return p * d // 2, p * d // 2, p * d // GROUP, p * d // GROUP


# A page keeps its positions in blocks of 16, a block in one piece for each of the 64 lanes of a wavefront (group g of 4, row r of 16).
# Keys: the row is the position, a piece holds a quarter of the head's features, two to a byte.  Values: a piece holds four consecutive
# positions of features r + 16 t, a byte those of features r + 32 u and r + 32 u + 16 of one position.  Scales: a byte e + 127 for each
# position and group.
def _parts(case, pool):
    """The pool [pages, kv_heads, bytes] as (keys [.., block, g, r, bytes], values [.., block, g, r, u, position of 4], scales [.., position,
    group] of each)."""
    n, d, blocks = _sections(case), case["head_dim"], case["page"] // 16
    k, v, ks, vs = pool[..., :sum(n)].split(n, -1)
    return (k.unflatten(-1, (blocks, 4, 16, d // 8)), v.unflatten(-1, (blocks, 4, 16, d // 32, 4)), ks.unflatten(-1, (case["page"], d // GROUP)),
            vs.unflatten(-1, (case["page"], d // GROUP)))


def _key_bytes(case, codes):
    """Codes [..., features] of a position -> [..., g, bytes]."""
    return (codes[..., 0::2] | codes[..., 1::2] << 4).unflatten(-1, (4, -1))


def _value_bytes(case, codes):
    """Codes [..., features] of a position -> [..., r, u]."""
    c = codes.unflatten(-1, (-1, 2, 16))
    return (c[..., 0, :] | c[..., 1, :] << 4).transpose(-1, -2)


def _prepared(case, seed, n_pages):
    """A pool whose pages hold keys and values N(0, 1), quantised group by group."""
    lead = (n_pages, case["kv_heads"])
    pool = torch.zeros(*lead, sum(_sections(case)), dtype=torch.uint8, device="cuda")
    k, v, ks, vs = _parts(case, pool)
    for i, scales in enumerate((ks, vs)):
        codes, exps = _quantised(_randn(seed, 10 + i, *lead, case["page"], case["head_dim"]), case["type"])
        scales.copy_(exps)
        codes = codes.unflatten(2, (-1, 16))
        if i == 0:
            k.copy_(_key_bytes(case, codes).transpose(-2, -3))
        else:
            v.copy_(_value_bytes(case, codes.unflatten(-2, (4, 4))).permute(0, 1, 2, 3, 5, 6, 4))
    return pool


def prepare(case, seed):
    s = _State()
    s.case = case
    if case["op"] == "build":
        _prepare_build(s, case, seed)
    else:
        _prepare_pages(s, case, seed)
    return s


def _own_pages(case, n_pages, max_ctx, pool):
    from paper_2502_20727_amd import binding as B
    t = {"bf16": B.SPD_BF16, "f16": B.SPD_F16}[case["type"]]
    cfg = B.spd_pages_config(case["q_heads"], case["kv_heads"], case["head_dim"], case["page"], n_pages, t, B.SPD_E2M1, max_ctx, ROPE_BASE)
    return B.DevicePages(cfg, torch.device("cuda"), pool=pool, rope=False)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prepare_pages(s, case, seed):
    s.positions, s.q_lens = _lengths(case)
    page, q, kv, d, t = case["page"], case["q_heads"], case["kv_heads"], case["head_dim"], TYPES[case["type"]]
    ends = s.ends = [p + n for p, n in zip(s.positions, s.q_lens)]
    held = [-(-e // page) for e in ends]
    n_pages = sum(held) + 3
    order = np.random.RandomState(int(seed) % (2 ** 31)).permutation(n_pages).astype(np.int32)
    # the page table of a program that hands out pages as they come free; unused entries are zero
    s.table = np.zeros((case["batch"], max(held)), dtype=np.int32)
    first = 0
    for b, n in enumerate(held):
        s.table[b, :n] = order[first:first + n]
        first += n
    max_ctx = -(-max(ends) // 32) * 32
    s.pool = _prepared(case, seed, n_pages)
    # of every new token: its sequence, its place in the chunk
    s.seq = torch.from_numpy(np.repeat(np.arange(case["batch"]), s.q_lens)).cuda()
    s.place = torch.from_numpy(np.concatenate([np.arange(n) for n in s.q_lens])).cuda()
    s.pos = torch.tensor(s.positions, device="cuda")
    s.table_dev = torch.from_numpy(s.table).cuda().long()
    tokens = sum(s.q_lens)
    if case["op"] == "attend":
        # the queries stand in the rows that the QKV projection wrote
        s.q = _randn(seed, 1, tokens, (q + 2 * kv) * d).to(t)[:, :q * d]
        s.out = torch.empty(tokens, q * d, dtype=t, device="cuda")
    else:
        if case["op"] == "store":
            s.qkv = _randn(seed, 1, tokens, (q + 2 * kv) * d).to(TYPES[case["in"]])
            theta = ROPE_BASE ** (-np.arange(d // 2, dtype=np.float64) / (d // 2))
            angle = np.arange(max_ctx, dtype=np.float64)[:, None] * theta
            s.rope = torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)).cuda()
            s.q_out = torch.empty(tokens, q * d, dtype=t, device="cuda")
            # what is read back: the pages that receive new tokens, from their first position on
            low = [p // page for p in s.positions]
        else:
            low = [0] * case["batch"]
        s.read_ends = [e - l * page for e, l in zip(ends, low)]
        entries = [-(-e // page) for e in s.read_ends]
        s.read_table = np.zeros((case["batch"], max(entries)), dtype=np.int32)
        for b, (l, n) in enumerate(zip(low, entries)):
            s.read_table[b, :n] = s.table[b, l:l + n]
        s.read_table_dev = torch.from_numpy(s.read_table).cuda().long()
        s.read_seq = torch.from_numpy(np.repeat(np.arange(case["batch"]), s.read_ends)).cuda()
        s.read_pos = torch.from_numpy(np.concatenate([np.arange(e) for e in s.read_ends])).cuda()
        s.k_out, s.v_out = (torch.empty(sum(s.read_ends), kv, d, dtype=t, device="cuda") for _ in range(2))
    if own:             # the handle of the pool and the plan of a step: made once and used by every layer of the model
        from paper_2502_20727_amd import binding as B
        s.pages = _own_pages(case, n_pages, max_ctx, s.pool)
        if case["op"] != "attend":
            s.read_plan = B.PagePlan(s.pages, [0] * case["batch"], s.read_ends, s.read_table)
        if case["op"] == "fetch":
            return
        if case["plan"] == "host":
            s.plan = B.PagePlan(s.pages, s.positions, s.q_lens, s.table, window=case["window"], sinks=case["sinks"])
        else:
            limits = B.spd_pages_limits(case["batch"], tokens, max(s.q_lens), s.table.shape[1], case["window"], case["sinks"])
            s.plan = B.DevicePlan(s.pages, limits)
            B.spd_pages_build(s.pages.ctx, s.plan, _int32(s.positions), _int32(s.q_lens), torch.from_numpy(s.table).cuda())


def _prepare_build(s, case, seed):
    positions, q_lens = _lengths(case)
    page, batch = case["page"], case["batch"]
    kept = [-(-p // page) for p in positions]
    ends = [p + max(n, 0) for p, n in zip(positions, q_lens)]
    need = sum(-(-e // page) - k for e, k in zip(ends, kept))
    s.n_pages = sum(kept) + need + 3
    order = np.random.RandomState(int(seed) % (2 ** 31)).permutation(s.n_pages).astype(np.int32)
    s.entries = max(-(-e // page) for e in ends) + 1
    table = np.full((batch, s.entries), -1, dtype=np.int32)
    first = 0
    for b, n in enumerate(kept):
        table[b, :n] = order[first:first + n]
        first += n
    # as many free pages as there are, or (beside requests that end) fewer than are needed: those that come back are used at once
    free = order[first:]
    s.free = torch.full((s.n_pages,), -1, dtype=torch.int32, device="cuda")
    s.free[:len(free)] = torch.from_numpy(free).cuda()
    back = sum(k for k, n in zip(kept, q_lens) if n < 0)
    s.n_free = _int32([max(need // 2, need - back) if back else len(free)])
    s.table = torch.from_numpy(table).cuda()
    s.positions, s.q_lens = _int32(positions), _int32(q_lens)
    s.tokens = sum(max(n, 0) for n in q_lens) + 5              # (a step with room to spare)
    s.longest = max(max(q_lens), 1)
    s.max_ctx = s.entries * page
    if own:             # everything that the steps of a server write to, made once
        from paper_2502_20727_amd import binding as B
        s.pages = _own_pages(case, s.n_pages, s.max_ctx, torch.empty(s.n_pages * case["kv_heads"] * sum(_sections(case)), dtype=torch.uint8, device="cuda"))
        s.plan = B.DevicePlan(s.pages, B.spd_pages_limits(batch, s.tokens, s.longest, s.entries, 0, 0))
        def ints(n, t=torch.int32):
            return torch.empty(n, dtype=t, device="cuda")
        s.n_free_out, s.positions_out, s.served, s.first_row = ints(1), ints(batch), ints(batch), ints(batch + 1)
        s.row_seq, s.row_pos, s.row_slot = ints(s.tokens), ints(s.tokens), ints(s.tokens, torch.int64)


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    return (_run_own if own else _run_plain)[s.case["op"]](s)


def _own_attend(s):
    from paper_2502_20727_amd import binding as B
    B.spd_pages_attention(s.pages.ctx, s.plan, s.q, s.pool, s.out, s.plan.workspace)
    return s.out


def _own_store(s):
    from paper_2502_20727_amd import binding as B
    B.spd_pages_write(s.pages.ctx, s.plan, s.qkv, s.rope, s.pool, s.q_out)
    B.spd_pages_read(s.pages.ctx, s.read_plan, s.pool, s.k_out, s.v_out)
    return s.q_out, s.k_out, s.v_out


def _own_fetch(s):
    from paper_2502_20727_amd import binding as B
    B.spd_pages_read(s.pages.ctx, s.read_plan, s.pool, s.k_out, s.v_out)
    return s.k_out, s.v_out


def _own_build(s):
    from paper_2502_20727_amd import binding as B
    B.spd_pages_build(s.pages.ctx, s.plan, s.positions, s.q_lens, s.table, free_pages=s.free, n_free=s.n_free, n_free_out=s.n_free_out,
                      positions_out=s.positions_out, served=s.served, first_row=s.first_row, row_seq=s.row_seq, row_pos=s.row_pos,
                      row_slot=s.row_slot)
    return {"table": s.table, "free": s.free, "n_free": s.n_free_out, "positions": s.positions_out, "served": s.served, "first_row": s.first_row,
            "row_seq": s.row_seq, "row_pos": s.row_pos, "row_slot": s.row_slot}


_run_own = {"attend": _own_attend, "store": _own_store, "fetch": _own_fetch, "build": _own_build}


def _quantised(x, type):
    """Codes [..., d] and scale bytes [..., d / 32] of rows x [..., d]."""
    lo, hi = EXPONENTS[type]
    x = x.unflatten(-1, (-1, GROUP))
    a = x.abs().amax(-1)
    m, k = torch.frexp(a)
    e = torch.where(a == 0, lo, (k - 3 + (m > 0.875)).clamp(lo, hi))
    y = torch.ldexp(x.abs(), -e[..., None])
    code = torch.signbit(x).to(torch.uint8) << 3
    # ties go to the code that is even
    for border, even in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += y >= border if even else y > border
    return code.flatten(-2), (e + 127).to(torch.uint8)


_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _pairs(codes):
    """Bytes -> the two values that each stands for, in a last dimension."""
    both = torch.tensor([[_VALUES[i & 15], _VALUES[i >> 4]] for i in range(256)], device="cuda")
    return both[codes.int()]


def _scaled(x, scales):
    """Values [..., d] by their groups' scales."""
    return (x.unflatten(-1, (-1, GROUP)) * torch.exp2(scales.float() - 127.0)[..., None]).flatten(-2)


def _gathered(case, pool, table):
    """Keys and values of every sequence in 32 bits, [batch, kv, positions, d], through the page table [batch, pages]."""
    k, v, ks, vs = (p[table] for p in _parts(case, pool))
    # [batch, pages, kv, block, g, r, byte, two] -> positions (block, r), features (g, byte, two)
    k = _pairs(k).permute(0, 1, 2, 3, 5, 4, 6, 7).flatten(5).flatten(3, 4)
    # [batch, pages, kv, block, g, r, u, place, two] -> positions (block, g, place), features (u, two, r)
    v = _pairs(v).permute(0, 1, 2, 3, 4, 7, 6, 8, 5).flatten(6).flatten(3, 5)
    return tuple(_scaled(x, f).transpose(1, 2).flatten(2, 3) for x, f in ((k, ks), (v, vs)))


def _visible(case, pos, q_len, n_keys):
    """[batch, q_len, keys]: which keys a query sees."""
    at = (pos[:, None] + torch.arange(q_len, device="cuda"))[:, :, None]
    key = torch.arange(n_keys, device="cuda")
    seen = key <= at
    if case["window"]:
        seen = seen & ((key > at - case["window"]) | (key < case["sinks"]))
    return seen


def _plain_attend(s):
    c = s.case
    q, kv, d, b, n = c["q_heads"], c["kv_heads"], c["head_dim"], c["batch"], max(s.q_lens)
    k, v = _gathered(c, s.pool, s.table_dev)
    padded = torch.zeros(b, n, q, d, device="cuda")
    padded[s.seq, s.place] = s.q.float().unflatten(-1, (q, d))
    rows = padded.view(b, n, kv, q // kv, d).permute(0, 2, 3, 1, 4).reshape(b, kv, (q // kv) * n, d)
    score = (torch.matmul(rows, k.transpose(2, 3).contiguous()) / math.sqrt(d)).view(b, q, n, -1)
    score.masked_fill_(~_visible(c, s.pos, n, k.shape[2])[:, None], float("-inf"))
    score = torch.exp_(score.sub_(score.amax(-1, keepdim=True)))
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(b, kv, -1, k.shape[2]), v).view(b, q, n, d) / total
    return o.transpose(1, 2)[s.seq, s.place].flatten(1).to(s.out.dtype)


def _rotated(x, cos, sin):
    lo, hi = x.chunk(2, -1)
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)


def _plain_store(s):
    c = s.case
    q, kv, d, page = c["q_heads"], c["kv_heads"], c["head_dim"], c["page"]
    x = s.qkv.unflatten(-1, (q + 2 * kv, d))
    at = s.pos[s.seq] + s.place
    cos, sin = s.rope[at].unbind(-1)
    keys = _rotated(x[:, q:q + kv].double(), cos[:, None].double(), sin[:, None].double())
    to, at = s.table_dev[s.seq, at // page], at % page
    k, v, ks, vs = _parts(c, s.pool)
    codes, ks[to, :, at] = _quantised(keys, c["type"])
    k[to, :, at // 16, :, at % 16] = _key_bytes(c, codes)
    codes, vs[to, :, at] = _quantised(x[:, q + kv:].float(), c["type"])
    v[to, :, at // 16, at % 16 // 4, :, :, at % 4] = _value_bytes(c, codes)
    return (_rotated(x[:, :q].float(), cos[:, None], sin[:, None]).flatten(1).to(s.q_out.dtype),) + _plain_fetch(s)


def _plain_fetch(s):
    return tuple(x[s.read_seq, :, s.read_pos].to(s.k_out.dtype) for x in _gathered(s.case, s.pool, s.read_table_dev))


def _plain_build(s):
    page, batch, tokens = s.case["page"], s.case["batch"], s.tokens
    pos, q, table = s.positions.long(), s.q_lens.long(), s.table
    rows = torch.where((q > 0) & (q <= s.longest), q, 0)
    last = rows.cumsum(0)
    first_row = torch.cat([torch.zeros_like(last[:1]), last]).clamp(max=tokens)
    fine = (pos >= 0) & (q >= -1) & (q <= s.longest) & (pos + q.clamp(min=0) <= s.max_ctx) & (last <= tokens)
    held = (pos + page - 1) // page
    # pages come back, in the requests' order, on top of the free ones ...
    back = torch.where(fine & (q == -1), held, 0)
    end = back.cumsum(0)
    entry = torch.arange(s.entries, device="cuda")
    place = torch.where(entry < back[:, None], (end - back + s.n_free)[:, None] + entry, s.n_pages)
    free = torch.cat([s.free, s.free.new_empty(1)]).scatter_(0, place.flatten(), table.flatten())[:-1]
    n_free = s.n_free + end[-1]
    # ... and new ones are taken from the top
    need = torch.where(fine & (q > 0), (pos + q + page - 1) // page - held, 0)
    end = need.cumsum(0)
    got = fine & ((end <= n_free) | (need == 0))
    nth = entry - held[:, None]
    fresh = (nth >= 0) & (nth < need[:, None]) & got[:, None]
    taken = free[(n_free - 1 - (end - need)[:, None] - nth).clamp(0, s.n_pages - 1)]
    table = table.copy_(torch.where(fresh, taken, table))
    valid = ((table >= 0) & (table < s.n_pages)) | (entry >= (held + need)[:, None])
    valid = valid.all(-1) | (q <= 0)
    good = got & valid
    served = torch.where(good, q.clamp(min=0), torch.where(got, -2, torch.where(fine, -3, -1)))
    # the rows' requests
    row = torch.arange(tokens, device="cuda")
    seq = torch.searchsorted(last, row, right=True)
    there = seq < batch
    b = seq.clamp(max=batch - 1)
    there &= good[b]
    at = pos[b] + row - (last - rows)[b]
    slot = table[b, (at // page).clamp(0, s.entries - 1)].long() * page + at % page
    row_seq, row_pos, row_slot = (torch.where(there, x, -1) for x in (b, at, slot))
    i32 = torch.int32
    return {"table": table, "free": s.free.copy_(free), "n_free": (n_free - torch.where(got, need, 0).sum()).to(i32),
            "positions": torch.where(good, torch.where(q == -1, 0, pos + q), pos).to(i32), "served": served.to(i32),
            "first_row": first_row.to(i32), "row_seq": row_seq.to(i32), "row_pos": row_pos.to(i32), "row_slot": row_slot}


_run_plain = {"attend": _plain_attend, "store": _plain_store, "fetch": _plain_fetch, "build": _plain_build}


# ------------------------------------------------------------------------------------------------ cost and reference

def work(case):
    op, page = case["op"], case["page"]
    size = {"f32": 4, "bf16": 2, "f16": 2}
    q, kv, d, t = case["q_heads"], case["kv_heads"], case["head_dim"], size[case["type"]]
    positions, q_lens = _lengths(case)
    row = kv * (d + 2 * d // GROUP)                # what a position of the cache holds
    tokens = sum(max(n, 0) for n in q_lens)
    if op == "build":
        # lengths in; kept entries checked, new ones taken and written, those that come back moved; per request and row what is written out
        entries = 0
        for p, n in zip(positions, q_lens):
            kept = -(-p // page)
            entries += 2 * kept if n < 0 else kept + 2 * (-(-(p + n) // page) - kept)
        return {"bytes": 4 * entries + case["batch"] * 20 + tokens * 16, "flops": 0}
    if op in ("store", "fetch"):
        held = sum(positions) + sum(q_lens) if op == "fetch" else sum(p % page + n for p, n in zip(positions, q_lens))
        moved = held * (row + 2 * kv * d * t)
        if op == "store":
            moved += tokens * ((q + 2 * kv) * d * size[case["in"]] + q * d * t + row)
        return {"bytes": moved, "flops": held * 2 * kv * d + (tokens * (q + 2 * kv) * d * 6 if op == "store" else 0)}
    w, sinks = case["window"], case["sinks"]
    keys = pairs = 0
    for p, n in zip(positions, q_lens):
        far = max(0, p - w + 1) if w else 0         # first position of the first query's window
        keys += p + n - far + min(sinks, far)
        for at in range(p, p + n):
            pairs += min(at + 1, w) + max(0, min(sinks, at + 1 - w)) if w else at + 1
    return {"bytes": keys * row + 2 * tokens * q * d * t, "flops": 4 * q * d * pairs}


def _exact_values(bytes_, steps):
    """Codes of 4 bits from the low and the high half of bytes, in 64 bits: sign, two bits of exponent, one of fraction."""
    c = torch.stack([bytes_ & 15, bytes_ >> 4], -1).double()
    sign, c = 1.0 - 2.0 * (c >= 8), c % 8
    e, m = torch.div(c, 2, rounding_mode="floor"), c % 2
    return sign * torch.where(e == 0, 0.5 * m, (1 + 0.5 * m) * 2.0 ** (e - 1)) * steps


def _exact_rows(case, s, b, table, end):
    """Keys and values of sequence b in 64 bits, [positions, kv, d]."""
    d, kv, out = case["head_dim"], case["kv_heads"], []
    k, v, ks, vs = (p[table[b]] for p in _parts(case, s.pool))
    n = k.shape[0]
    at = torch.arange(n * case["page"], device="cuda")
    page, at = at // case["page"], at % case["page"]
    feature = torch.arange(d, device="cuda")
    quarter = d // 4
    both = (_exact_values(k, 1.0)[page, :, at // 16, :, at % 16],            # [positions, kv, g, byte, two]
            _exact_values(v, 1.0)[page, :, at // 16, at % 16 // 4, :, :, at % 4])     # [positions, kv, r, u, two]
    k = both[0][:, :, feature // quarter, feature % quarter // 2, feature % 2]
    v = both[1][:, :, feature % 16, feature // 32, feature % 32 // 16]
    for x, f in ((k, ks), (v, vs)):
        step = 2.0 ** (f[page, :, at].double() - 127)
        out.append((x * step[:, :, feature // GROUP])[:end])
    return out


def _exact_attend(case, s):
    q, kv, d, out, first = case["q_heads"], case["kv_heads"], case["head_dim"], [], 0
    for b, (p, n) in enumerate(zip(s.positions, s.q_lens)):
        k, v = _exact_rows(case, s, b, s.table_dev, p + n)
        x = s.q[first:first + n].double().unflatten(-1, (q, d))
        first += n
        at, key = torch.arange(p, p + n, device="cuda")[:, None], torch.arange(p + n, device="cuda")
        hidden = key > at
        if case["window"]:
            hidden |= (key <= at - case["window"]) & (key >= case["sinks"])
        o = torch.empty(n, q, d, dtype=torch.float64, device="cuda")
        for j in range(q):
            g = j // (q // kv)
            o[:, j] = torch.softmax((x[:, j] @ k[:, g].t() / d ** 0.5).masked_fill_(hidden, float("-inf")), -1) @ v[:, g]
        out.append(o.flatten(1))
    return torch.cat(out)


def _exact_group(x, type):
    """Rows [..., d] as 4 bits hold them."""
    lo, hi = EXPONENTS[type]
    x = x.unflatten(-1, (-1, GROUP))
    e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 7)).clamp(lo, hi)
    step = 2.0 ** e
    # (log2 rounds: the exponent below or above, if that is the least)
    step = torch.where((x.abs().amax(-1, keepdim=True) <= 3.5 * step) & (e > lo), step / 2, step)
    step = torch.where((x.abs().amax(-1, keepdim=True) > 7 * step) & (e < hi), step * 2, step)
    y = x.abs() / step
    y = torch.where(y < 2, torch.round(y * 2) / 2, torch.where(y < 4, torch.round(y), (torch.round(y / 2) * 2).clamp(max=6)))
    return (torch.sign(x) * y * step).flatten(-2)


def _exact_store(case, s):
    q, kv, d, page = case["q_heads"], case["kv_heads"], case["head_dim"], case["page"]
    half, rotated, keys, values, first = d // 2, [], [], [], 0
    for b, (p, n) in enumerate(zip(s.positions, s.q_lens)):
        x = s.qkv[first:first + n].double().unflatten(-1, (q + 2 * kv, d))
        first += n
        cos, sin = (f[:, None] for f in s.rope[p:p + n].double().unbind(-1))
        turn = torch.cat([x[..., :half] * cos - x[..., half:] * sin, x[..., half:] * cos + x[..., :half] * sin], -1)
        rotated.append(turn[:, :q].flatten(1))
        old = _exact_rows(case, s, b, s.read_table_dev, p % page)       # what the first page held
        keys += [old[0], _exact_group(turn[:, q:q + kv], case["type"])]
        values += [old[1], _exact_group(x[:, q + kv:], case["type"])]
    return torch.cat(rotated), torch.cat(keys), torch.cat(values)


def _exact_fetch(case, s):
    both = [_exact_rows(case, s, b, s.read_table_dev, e) for b, e in enumerate(s.read_ends)]
    return tuple(torch.cat([x[i] for x in both]) for i in range(2))


def _exact_build(case, s):
    """Request by request, with a stack."""
    page, table, free = case["page"], s.table.cpu().numpy().copy(), s.free.cpu().numpy().copy()
    pos, q, top = s.positions.tolist(), s.q_lens.tolist(), int(s.n_free)
    for b in range(case["batch"]):
        for i in range(-(-pos[b] // page) if q[b] == -1 else 0):
            free[top], top = table[b, i], top + 1
    positions, served, first_row, seq, at, slot = [], [], [0], [], [], []
    for b in range(case["batch"]):
        n = max(q[b], 0)
        new = range(-(-pos[b] // page), -(-(pos[b] + n) // page))
        for i in new:
            top -= 1
            table[b, i] = free[top]
        served.append(n)
        positions.append(0 if q[b] == -1 else pos[b] + n)
        first_row.append(first_row[-1] + n)
        for p in range(pos[b], pos[b] + n):
            seq.append(b)
            at.append(p)
            slot.append(int(table[b, p // page]) * page + p % page)
    rest = [-1] * (s.tokens - len(seq))
    return {"table": table, "free": free, "n_free": np.array([top], dtype=np.int32), "positions": np.array(positions, dtype=np.int32),
            "served": np.array(served, dtype=np.int32), "first_row": np.array(first_row, dtype=np.int32),
            "row_seq": np.array(seq + rest, dtype=np.int32), "row_pos": np.array(at + rest, dtype=np.int32), "row_slot": np.array(slot + rest)}


def exact(case, seed):
    return {"attend": _exact_attend, "store": _exact_store, "fetch": _exact_fetch, "build": _exact_build}[case["op"]](case, prepare(case, seed))
