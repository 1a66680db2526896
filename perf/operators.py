"""The 8-bit serving operators and what is watched of their speed: a paged KV cache that is quantised as it is written and read
back, attention of chunks of new tokens (single ones among them) over its pages, with or without a sliding window and sinks, rows
brought to 8-bit integers behind a norm, a SwiGLU product or as they are, and the product of 8-bit rows with 8-bit weights.
Head counts and widths are those of one tensor-parallel rank, or of the whole model, of paper_2502_20727_amd/workloads.py.

Every operator stands here three times: as a user calls it (`own`), in a plain form of elementary torch operations in 32 bits, and
(exact) from its definition in 64 bits.

A case is a dict; `op` says which operator:
  "attend"   q_heads, kv_heads, head_dim, page, type (queries, output), cache ("e4m3" | the same 16-bit type), batch, q_len, ctx
             (positions before the chunk), ragged (chunks and contexts differ), window, sinks
  "store"    the same geometry: queries and keys rotated, keys and values quantised into their pages; in: type of the input rows
  "fetch"    the same geometry: everything the sequences hold, back as dense rows of `type`
  "norm"     rows, cols, type, add (a second summand, whose sum with the first is written too)
  "rows" | "swiglu"   rows, cols, type
  "product"  rows, k, n, type (output), add (a summand of the output's type)
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
ROPE_BASE = 10000.0
E4M3_MAX = 448.0
LEAST = 2.0 ** -90          # the quantisers' least largest magnitude of a row


def _pages(name, op, heads, batch, q_len, ctx, type="bf16", cache="e4m3", page=64, ragged=False, window=0, sinks=0, **more):
    q, kv, d = heads
    return {"name": name, "op": op, "q_heads": q, "kv_heads": kv, "head_dim": d, "page": page, "type": type, "cache": cache,
            "batch": batch, "q_len": q_len, "ctx": ctx, "ragged": ragged, "window": window, "sinks": sinks, **more}


def listed():
    return [
        # interactive decoding of one sequence on an eighth of the 7B model: latency
        _pages("attend-7b-step-b1-ctx2048", "attend", (4, 4, 128), 1, 1, 2047),
        # continuous batching on an eighth of the 70B model: 48 sequences of different lengths, one new token each
        _pages("attend-70b-steps-b48-ragged", "attend", (8, 1, 128), 48, 1, 16000, ragged=True),
        # chunks of three prompts of a 13B rank behind long contexts, window of 2048 and four sinks, 16-bit pages, odd lengths
        _pages("attend-13b-chunks-3x333-window", "attend", (5, 5, 128), 3, 333, 5001, type="f16", cache="f16", page=16,
               ragged=True, window=2048, sinks=4),
        # four prompts of 2048 tokens, all heads of the 70B model on one GPU
        _pages("attend-70b-prompts-4x2048", "attend", (64, 8, 128), 4, 2048, 0),
        # a decode step of 16 sequences puts away its keys and values
        _pages("store-70b-steps-b16", "store", (8, 1, 128), 16, 1, 4095, **{"in": "bf16"}),
        # four prompts of 2048 tokens do, all heads of the 70B model
        _pages("store-70b-prompts-4x2048", "store", (64, 8, 128), 4, 2048, 0, **{"in": "bf16"}),
        # sequences handed to another pool or another program: 16 contexts of about 4096 positions read back
        _pages("fetch-70b-b16-ragged", "fetch", (8, 1, 128), 16, 1, 4095, ragged=True),
        # the norm of a decode step of 16 sequences, behind the partial attention output that an SPD block folds in
        {"name": "norm-16x8192-f32-add", "op": "norm", "rows": 16, "cols": 8192, "type": "f32", "add": True},
        # the same of four prompts of 2048 tokens, residual stream kept in 16 bits
        {"name": "norm-8192x8192-bf16-add", "op": "norm", "rows": 8192, "cols": 8192, "type": "bf16", "add": True},
        # gate and up projection of an eighth of the 70B model, decode step of 16 sequences
        {"name": "product-16x8192x7168", "op": "product", "rows": 16, "k": 8192, "n": 7168, "type": "bf16", "add": False},
        # down projection of an eighth of the 13B model for an odd prompt, onto the partial attention output
        {"name": "product-333x1728x5120-add", "op": "product", "rows": 333, "k": 1728, "n": 5120, "type": "f32", "add": True},
        # gate and up projection of four prompts of 2048 tokens
        {"name": "product-8192x8192x7168", "op": "product", "rows": 8192, "k": 8192, "n": 7168, "type": "bf16", "add": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choices(["attend", "store", "fetch", "norm", "rows", "swiglu", "product"], [5, 2, 1, 2, 1, 1, 4])[0]
    if op in ("attend", "store", "fetch"):
        heads = rng.choice([(8, 1, 128), (64, 8, 128), (4, 4, 128), (5, 5, 128), (10, 10, 128), (40, 40, 128), (4, 4, 64), (12, 4, 64)])
        step = rng.random() < (0.5 if op != "fetch" else 1.0)
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
        c = _pages("", op, heads, batch, q_len, ctx, type=type, cache=rng.choice(["e4m3", "e4m3", type]),
                   page=rng.choice([16, 32, 64, 128]), ragged=rng.random() < 0.6, window=window,
                   sinks=rng.choice([0, 4, rng.randrange(1, 100)]) if window else 0, **more)
    elif op == "product":
        rows = _log_int(rng, 1, 8192)
        k, n = rng.choice([(8192, 1280), (1024, 8192), (8192, 7168), (3584, 8192), (5120, 1920), (640, 5120), (5120, 3456),
                           (1728, 5120), (4096, 1536), (512, 4096), (4096, 2752), (1376, 4096), (256, 688), (688, 257),
                           (16 * rng.randrange(1, 300), rng.randrange(1, 5000))])
        c = {"op": op, "rows": rows, "k": k, "n": n, "type": rng.choice(["bf16", "f32", "f16"]), "add": rng.random() < 0.4}
    else:
        cols = rng.choice([8192, 5120, 4096, 3584, 1728, 1376, 1024, 256, 688, rng.randrange(1, 9000)])
        c = {"op": op, "rows": _log_int(rng, 1, 8192), "cols": cols, "type": rng.choice(["f32", "bf16", "f16"])}
        if op == "norm":
            c["add"] = rng.random() < 0.7
    c.pop("name", None)
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed, key):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + key * 7919) % (2 ** 62))
    return g


def _randn(seed, key, *shape):
    return torch.randn(*shape, generator=_generator(seed, key), device="cuda")


def _ints(seed, key, *shape):
    """8-bit codes as a quantiser leaves them: normal values whose largest, four deviations off, stands at 127."""
    return (_randn(seed, key, *shape) * 32.0).round_().clamp_(-127, 127).to(torch.int8)


def _lengths(case):
    """(positions before the chunk, new tokens) of each sequence: part of the case, whatever the seed."""
    b, n, ctx = case["batch"], case["q_len"], case["ctx"]
    if not case["ragged"]:
        return [ctx] * b, [n] * b
    r = random.Random(b * 1000003 + n * 7919 + ctx)
    return ([ctx] + [r.randint(ctx // 4, ctx) for _ in range(b - 1)], [n] + [r.randint(max(1, n // 2), n) for _ in range(b - 1)])


class _State:
    pass


def _width(case):
    return 1 if case["cache"] == "e4m3" else 2


def _head_bytes(case):
    """Bytes of one head's share of a page: its keys, its values, a scale in 32 bits for each of them."""
    return case["page"] * (2 * case["head_dim"] * _width(case) + 8)


def _parts(case, pool):
    """The pool [pages, kv_heads, bytes] as (codes of the keys, codes of the values, scales of the keys, of the values)."""
    p, n = case["page"], case["page"] * case["head_dim"] * _width(case)
    t = torch.float8_e4m3fn if case["cache"] == "e4m3" else TYPES[case["cache"]]
    return (pool[..., :n].view(t), pool[..., n:2 * n].view(t), pool[..., 2 * n:2 * n + 4 * p].view(torch.float32),
            pool[..., 2 * n + 4 * p:].view(torch.float32))


# A page keeps its positions in blocks of 16, a block in pieces of 16 bytes, in the order in which the 64 lanes of a wavefront take
# them up (group g of 4, row r of 16).  Keys: the row is the position, a piece holds consecutive features.  Values: the row is one of
# 16 features, a piece holds four consecutive positions of each of several such features.
def _key_view(case, t):
    e = 16 // _width(case)
    return t.unflatten(-1, (case["page"] // 16, case["head_dim"] // (4 * e), 4, 16, e))


def _value_view(case, t):
    e = 16 // _width(case)
    return t.unflatten(-1, (case["page"] // 16, case["head_dim"] // (4 * e), 4, 16, e // 4, 4))


def _natural(case, keys, values):
    """Pieces of pages [..., kv, codes] -> [..., kv, position, feature]."""
    k, v = _key_view(case, keys), _value_view(case, values)
    n = k.dim() - 5
    lead = list(range(n))
    k = k.permute(lead + [n, n + 3, n + 1, n + 2, n + 4])
    v = v.permute(lead + [n, n + 2, n + 5, n + 1, n + 4, n + 3])
    return k.flatten(n, n + 1).flatten(n + 1), v.flatten(n, n + 2).flatten(n + 1)


def _laid_out(case, k, v):
    """The inverse: natural [..., position, feature] -> codes in the order of the page."""
    e, n = 16 // _width(case), k.dim() - 2
    lead, blocks = list(range(n)), case["page"] // 16
    k = k.unflatten(-1, (-1, 4, e)).unflatten(n, (blocks, 16)).permute(lead + [n, n + 2, n + 3, n + 1, n + 4])
    v = v.unflatten(-1, (-1, e // 4, 16)).unflatten(n, (blocks, 4, 4)).permute(lead + [n, n + 3, n + 1, n + 5, n + 4, n + 2])
    return k.flatten(n), v.flatten(n)


def _filled_pool(case, seed, n_pages):
    """A pool whose pages hold keys and values N(0, 1), quantised row by row."""
    shape = (n_pages, case["kv_heads"], case["page"], case["head_dim"])
    pool = torch.zeros(n_pages, case["kv_heads"], _head_bytes(case), dtype=torch.uint8, device="cuda")
    parts, codes = _parts(case, pool), []
    for i in range(2):
        x = _randn(seed, 10 + i, *shape)
        if case["cache"] == "e4m3":
            a = x.abs().amax(-1, keepdim=True)
            parts[2 + i].copy_((a / E4M3_MAX).squeeze(-1))
            codes.append((x * (E4M3_MAX / a)).to(torch.float8_e4m3fn))
        else:
            parts[2 + i].fill_(1.0)
            codes.append(x.to(TYPES[case["cache"]]))
    raw = torch.uint8 if case["cache"] == "e4m3" else torch.int16
    for part, laid in zip(parts, _laid_out(case, codes[0].view(raw), codes[1].view(raw))):
        part.view(raw).copy_(laid)
    return pool


def _rope(case, positions):
    """cos and sin of the rotary angles of `positions`, in 64 bits: far positions leave 32 bits no digits."""
    half = case["head_dim"] // 2
    theta = ROPE_BASE ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    a = positions.to(torch.float64)[:, None] * theta
    return a.cos(), a.sin()


def prepare(case, seed):
    s = _State()
    s.case = case
    if case["op"] in ("attend", "store", "fetch"):
        _prepare_pages(s, case, seed)
    elif case["op"] == "product":
        # 8-bit rows as the quantisers leave them, weights in 8 bits with a scale for each output channel
        s.a, s.w = _ints(seed, 1, case["rows"], case["k"]), _ints(seed, 2, case["k"], case["n"])
        s.a_scale = 0.02 + 0.02 * torch.rand(case["rows"], generator=_generator(seed, 3), device="cuda")
        s.w_scale = (0.5 + torch.rand(case["n"], generator=_generator(seed, 4), device="cuda")) * (0.02 / 32)
        t = TYPES[case["type"]]
        s.add = _randn(seed, 5, case["rows"], case["n"]).to(t) if case["add"] else None
        if own:         # the weights are laid out once, when they are loaded
            from paper_2502_20727_amd import binding as B
            packed = B.spd_q8_pack_codes(s.w.cpu().numpy(), s.w_scale.cpu().numpy())
            s.packed = torch.from_numpy(packed).cuda()
            s.out = torch.empty(case["rows"], case["n"], dtype=t, device="cuda")
            s.workspace = torch.empty(B.spd_q8_matmul_workspace(case["rows"], case["k"], case["n"]), dtype=torch.uint8, device="cuda")
    else:
        t, rows, cols = TYPES[case["type"]], case["rows"], case["cols"]
        s.x = _randn(seed, 1, rows, cols * (2 if case["op"] == "swiglu" else 1)).to(t)
        s.add = (0.3 * _randn(seed, 2, rows, cols)).to(t) if case.get("add") else None
        s.gain = 1.0 + 0.02 * _randn(seed, 3, cols)
        s.sum = torch.empty(rows, cols, dtype=t, device="cuda") if case.get("add") else None
        s.codes = torch.empty(rows, cols, dtype=torch.int8, device="cuda")
        s.scale = torch.empty(rows, dtype=torch.float32, device="cuda")
        s.values = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    return s


def _prepare_pages(s, case, seed):
    s.positions, s.q_lens = _lengths(case)
    page, q, kv, d, t = case["page"], case["q_heads"], case["kv_heads"], case["head_dim"], TYPES[case["type"]]
    ends = [p + n for p, n in zip(s.positions, s.q_lens)]
    held = [-(-e // page) for e in ends]
    n_pages = sum(held) + 3
    order = np.random.RandomState(int(seed) % (2 ** 31)).permutation(n_pages).astype(np.int32)
    # the page table of a program that hands out pages as they come free; unused entries are zero
    s.table = np.zeros((case["batch"], max(held)), dtype=np.int32)
    first = 0
    for b, n in enumerate(held):
        s.table[b, :n] = order[first:first + n]
        first += n
    s.max_ctx = -(-max(ends) // 32) * 32
    s.pool = _filled_pool(case, seed, n_pages)
    # of every new token: its sequence, its place in the chunk, its position
    seq = np.repeat(np.arange(case["batch"]), s.q_lens)
    place = np.concatenate([np.arange(n) for n in s.q_lens])
    s.seq, s.place = torch.from_numpy(seq).cuda(), torch.from_numpy(place).cuda()
    s.pos = torch.tensor(s.positions, device="cuda")
    s.ends = torch.tensor(ends, device="cuda")
    s.table_dev = torch.from_numpy(s.table).cuda().long()
    s.kept = [e for e in ends]
    tokens = len(seq)
    if case["op"] == "store":
        s.qkv = _randn(seed, 1, tokens, (q + 2 * kv) * d).to(TYPES[case["in"]])
        s.cos, s.sin = (x.float() for x in _rope(case, torch.arange(s.max_ctx, device="cuda")))
        s.q_out = torch.empty(tokens, q * d, dtype=t, device="cuda")
    elif case["op"] == "attend":
        # the queries stand in the rows that the QKV projection wrote
        s.q = _randn(seed, 1, tokens, (q + 2 * kv) * d).to(t)[:, :q * d]
        s.out = torch.empty(tokens, q * d, dtype=t, device="cuda")
    else:
        s.k_out, s.v_out = (torch.empty(sum(ends), kv, d, dtype=t, device="cuda") for _ in range(2))
        s.held_seq = torch.from_numpy(np.repeat(np.arange(case["batch"]), ends)).cuda()
        s.held_pos = torch.from_numpy(np.concatenate([np.arange(e) for e in ends])).cuda()
    if own:             # the handle of the pool and the plan of a step: made once and used by every layer of the model
        from paper_2502_20727_amd import binding as B
        types = {"f32": B.SPD_F32, "bf16": B.SPD_BF16, "f16": B.SPD_F16, "e4m3": B.SPD_E4M3}
        cfg = B.spd_pages_config(q, kv, d, page, n_pages, types[case["type"]], types[case["cache"]], s.max_ctx, ROPE_BASE)
        s.pages = B.DevicePages(cfg, torch.device("cuda"), pool=s.pool)
        s.plan = B.PagePlan(s.pages, s.positions, s.q_lens, s.table, window=case["window"], sinks=case["sinks"])


# ------------------------------------------------------------------------------------------------ one pass

def run(s):
    return (_run_own if own else _run_plain)[s.case["op"]](s)


def _own_attend(s):
    from paper_2502_20727_amd import binding as B
    B.spd_pages_attention(s.pages.ctx, s.plan, s.q, s.pool, s.out, s.plan.workspace)
    return s.out


def _own_store(s):
    from paper_2502_20727_amd import binding as B
    B.spd_pages_write(s.pages.ctx, s.plan, s.qkv, s.pages.rope, s.pool, s.q_out)
    return (s.q_out,) + _parts(s.case, s.pool)


def _own_fetch(s):
    from paper_2502_20727_amd import binding as B
    B.spd_pages_read(s.pages.ctx, s.plan, s.pool, s.k_out, s.v_out)
    return s.k_out, s.v_out


def _values(s):
    """What the codes stand for, in 16 bits."""
    return torch.mul(s.codes, s.scale[:, None], out=s.values)


def _own_norm(s):
    from paper_2502_20727_amd import binding as B
    B.spd_q8_norm(s.x, s.add, s.gain, EPS, s.sum, s.codes, s.scale)
    return s.sum, _values(s), s.scale


def _own_rows(s):
    from paper_2502_20727_amd import binding as B
    B.spd_q8_rows(s.x, s.codes, s.scale)
    return _values(s), s.scale


def _own_swiglu(s):
    from paper_2502_20727_amd import binding as B
    B.spd_q8_swiglu(s.x, s.codes, s.scale)
    return _values(s), s.scale


def _own_product(s):
    from paper_2502_20727_amd import binding as B
    B.spd_q8_matmul(s.a, s.a_scale, s.packed, s.case["n"], s.add, s.out, s.workspace)
    return s.out


_run_own = {"attend": _own_attend, "store": _own_store, "fetch": _own_fetch, "norm": _own_norm, "rows": _own_rows,
            "swiglu": _own_swiglu, "product": _own_product}


def _gathered(case, pool, table):
    """Keys and values of every sequence in 32 bits, [batch, kv, positions, d], through the page table [batch, pages]."""
    k8, v8, ks, vs = _parts(case, pool)
    k, v = _natural(case, k8[table].float(), v8[table].float())
    k, v = k * ks[table][..., None], v * vs[table][..., None]
    return k.transpose(1, 2).flatten(2, 3), v.transpose(1, 2).flatten(2, 3)


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
    score = (torch.matmul(rows, k.transpose(2, 3)) / math.sqrt(d)).view(b, q, n, -1)
    score.masked_fill_(~_visible(c, s.pos, n, k.shape[2])[:, None], float("-inf"))
    score = torch.exp_(score.sub_(score.amax(-1, keepdim=True)))
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(b, kv, -1, k.shape[2]), v).view(b, q, n, d) / total
    return o.transpose(1, 2)[s.seq, s.place].flatten(1).to(s.out.dtype)


def _rotated(x, cos, sin):
    lo, hi = x.chunk(2, -1)
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)


def _scatter(case, keys, values, page, at, k, v):
    """Rows k, v [tokens, kv, d] into the codes of the pages, at positions `at` of `page`."""
    e = 16 // _width(case)
    _key_view(case, keys)[page, :, at // 16, :, :, at % 16] = k.unflatten(-1, (-1, 4, e))
    _value_view(case, values)[page, :, at // 16, :, at % 16 // 4, :, :, at % 4] = \
        v.unflatten(-1, (-1, e // 4, 16)).transpose(-1, -2)


def _plain_store(s):
    c = s.case
    q, kv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    x = s.qkv.float().unflatten(-1, (q + 2 * kv, d))
    at = s.pos[s.seq] + s.place
    cos, sin = s.cos[at][:, None], s.sin[at][:, None]
    page = s.table_dev[s.seq, at // c["page"]]
    at = at % c["page"]
    parts, codes = _parts(c, s.pool), []
    for i, row in enumerate((_rotated(x[:, q:q + kv], cos, sin), x[:, q + kv:])):
        if c["cache"] == "e4m3":
            a = row.abs().amax(-1, keepdim=True).clamp_(min=LEAST)
            parts[2 + i][page, :, at] = (a / E4M3_MAX).squeeze(-1)
            codes.append((row * (E4M3_MAX / a)).to(torch.float8_e4m3fn).view(torch.uint8))
        else:
            parts[2 + i][page, :, at] = 1.0
            codes.append(row.to(TYPES[c["cache"]]).view(torch.int16))
    _scatter(c, parts[0].view(codes[0].dtype), parts[1].view(codes[0].dtype), page, at, *codes)
    return (_rotated(x[:, :q], cos, sin).flatten(1).to(s.q_out.dtype),) + parts


def _plain_fetch(s):
    k, v = _gathered(s.case, s.pool, s.table_dev)
    return tuple(x[s.held_seq, :, s.held_pos].to(s.k_out.dtype) for x in (k, v))


def _codes_of(rows):
    """The 8-bit quantiser: values and scale of each row."""
    a = rows.abs().amax(-1, keepdim=True).clamp(min=LEAST)
    return torch.round(rows * (127.0 / a)) * (a / 127.0), (a / 127.0).squeeze(-1)


def _plain_norm(s):
    x = s.x.float()
    if s.add is not None:
        x = x + s.add.float()
    y, scale = _codes_of(x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * s.gain)
    return x.to(s.x.dtype) if s.add is not None else None, y.to(torch.bfloat16), scale


def _plain_rows(s):
    y, scale = _codes_of(s.x.float())
    return y.to(torch.bfloat16), scale


def _plain_swiglu(s):
    g, u = s.x.float().chunk(2, -1)
    y, scale = _codes_of(g / (1.0 + torch.exp(-g)) * u)
    return y.to(torch.bfloat16), scale


def _plain_product(s):
    out = torch.matmul(s.a.float(), s.w.float()) * s.a_scale[:, None] * s.w_scale
    if s.add is not None:
        out = out + s.add.float()
    return out.to(TYPES[s.case["type"]])


_run_plain = {"attend": _plain_attend, "store": _plain_store, "fetch": _plain_fetch, "norm": _plain_norm, "rows": _plain_rows,
              "swiglu": _plain_swiglu, "product": _plain_product}


# ------------------------------------------------------------------------------------------------ cost and reference

def work(case):
    op = case["op"]
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if op == "product":
        m, k, n = case["rows"], case["k"], case["n"]
        return {"bytes": m * k + k * n + 4 * (m + n) + m * n * size[case["type"]] * (2 if case["add"] else 1), "flops": 2 * m * k * n}
    if op in ("norm", "rows", "swiglu"):
        m, n, t = case["rows"], case["cols"], size[case["type"]]
        inputs = 2 if op == "swiglu" or case.get("add") else 1
        sums = 1 if case.get("add") else 0
        return {"bytes": m * n * (t * (inputs + sums) + 1) + 4 * m + (4 * n if op == "norm" else 0), "flops": 8 * m * n}
    q, kv, d, t = case["q_heads"], case["kv_heads"], case["head_dim"], size[case["type"]]
    positions, q_lens = _lengths(case)
    row = kv * (2 * d * _width(case) + 8)          # what a position of the cache holds
    if op == "store":
        tokens = sum(q_lens)
        return {"bytes": tokens * ((q + 2 * kv) * d * size[case["in"]] + q * d * t + row), "flops": tokens * (q + 2 * kv) * d * 6}
    if op == "fetch":
        held = sum(positions) + sum(q_lens)
        return {"bytes": held * (row + 2 * kv * d * t), "flops": held * 2 * kv * d}
    w, sinks = case["window"], case["sinks"]
    keys = pairs = 0
    for p, n in zip(positions, q_lens):
        far = max(0, p - w + 1) if w else 0         # first position of the first query's window
        keys += p + n - far + min(sinks, far)
        for at in range(p, p + n):
            pairs += min(at + 1, w) + max(0, min(sinks, at + 1 - w)) if w else at + 1
    return {"bytes": keys * row + 2 * sum(q_lens) * q * d * t, "flops": 4 * q * d * pairs}


def _exact_rows(rows):
    a = rows.abs().amax(-1, keepdim=True).clamp(min=LEAST)
    return torch.round(rows * 127 / a) * a / 127, (a / 127).squeeze(-1)


def _exact_sequence(case, s, b):
    """Keys and values of sequence b in 64 bits, [kv, positions, d]."""
    k8, v8, ks, vs = (p[s.table_dev[b]] for p in _parts(case, s.pool))
    k, v = _natural(case, k8.double(), v8.double())
    end = s.kept[b]
    return tuple((x * f.double()[..., None]).transpose(0, 1).flatten(1, 2)[:, :end] for x, f in ((k, ks), (v, vs)))


def _exact_attend(case, s):
    q, kv, d, out, first = case["q_heads"], case["kv_heads"], case["head_dim"], [], 0
    for b, (p, n) in enumerate(zip(s.positions, s.q_lens)):
        k, v = _exact_sequence(case, s, b)
        x = s.q[first:first + n].double().unflatten(-1, (q, d))
        first += n
        at, key = torch.arange(p, p + n, device="cuda")[:, None], torch.arange(p + n, device="cuda")
        hidden = key > at
        if case["window"]:
            hidden |= (key <= at - case["window"]) & (key >= case["sinks"])
        o = torch.empty(n, q, d, dtype=torch.float64, device="cuda")
        for j in range(q):
            g = j // (q // kv)
            o[:, j] = torch.softmax((x[:, j] @ k[g].t() / d ** 0.5).masked_fill_(hidden, float("-inf")), -1) @ v[g]
        out.append(o.flatten(1))
    return torch.cat(out)


def _exact_store(case, s):
    q, kv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    parts = [p.double() for p in _parts(case, s.pool)]
    rotated, first = [], 0
    for b, (p, n) in enumerate(zip(s.positions, s.q_lens)):
        x = s.qkv[first:first + n].double().unflatten(-1, (q + 2 * kv, d))
        first += n
        at = torch.arange(p, p + n, device="cuda")
        cos, sin = (f[:, None] for f in _rope(case, at))
        half = d // 2
        turn = torch.cat([x[..., :half] * cos - x[..., half:] * sin, x[..., half:] * cos + x[..., :half] * sin], -1)
        rotated.append(turn[:, :q].flatten(1))
        page, at = s.table_dev[b, at // case["page"]], at % case["page"]
        codes = []
        for i, row in enumerate((turn[:, q:q + kv], x[:, q + kv:])):
            if case["cache"] == "e4m3":
                a = row.abs().amax(-1, keepdim=True).clamp(min=LEAST)
                parts[2 + i][page, :, at] = (a / E4M3_MAX).squeeze(-1)
                codes.append((row * E4M3_MAX / a).float().to(torch.float8_e4m3fn).double())
            else:
                parts[2 + i][page, :, at] = 1.0
                codes.append(row)
        _scatter(case, parts[0], parts[1], page, at, *codes)
    return (torch.cat(rotated),) + tuple(parts)


def _exact_fetch(case, s):
    both = [_exact_sequence(case, s, b) for b in range(case["batch"])]
    return tuple(torch.cat([x[i].transpose(0, 1) for x in both]) for i in range(2))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "attend":
        return _exact_attend(case, s)
    if op == "store":
        return _exact_store(case, s)
    if op == "fetch":
        return _exact_fetch(case, s)
    if op == "product":
        total = (s.a.double() @ s.w.double()) * s.a_scale.double()[:, None] * s.w_scale.double()
        return total if s.add is None else total + s.add.double()
    x = s.x.double()
    if op == "rows":
        return _exact_rows(x)
    if op == "swiglu":
        g, u = x.chunk(2, -1)
        return _exact_rows(g * torch.sigmoid(g) * u)
    if s.add is not None:
        x = x + s.add.double()
    y, scale = _exact_rows(x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * s.gain.double())
    return x if s.add is not None else None, y, scale
