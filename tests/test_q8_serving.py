"""The 8-bit serving operators (include/spd_q8.h): plans, packers and refusals on the CPU, numerics on the GPU against plain
computations in 64 bits.

Tolerances count roundings: u = torch.finfo(t).eps / 2 of a value rounded to type t, half a step of a quantised one."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2502_20727_amd import binding as B

gpu_test = pytest.mark.gpu
T16 = {B.SPD_BF16: torch.bfloat16, B.SPD_F16: torch.float16}
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}
U32 = 2.0 ** -24
LEAST = 2.0 ** -90


def config(q=8, kv=2, d=128, page=32, n_pages=40, dtype=B.SPD_BF16, cache=B.SPD_E4M3, max_ctx=1024, base=10000.0):
    return B.spd_pages_config(q, kv, d, page, n_pages, dtype, cache, max_ctx, base)


# ------------------------------------------------------------------------------------------ the pool, read from its bytes

def natural(cfg, pool):
    """(keys, values) of a pool (bytes, CPU) as [pages, kv, position, d] float64, code * scale; and the scales."""
    w = 1 if cfg.cache_dtype == B.SPD_E4M3 else 2
    p, d, kv = cfg.page_size, cfg.head_dim, cfg.n_kv_heads
    n = p * d * w
    raw = pool.view(cfg.n_pages, kv, p * (2 * d * w + 8))
    t = torch.float8_e4m3fn if w == 1 else T16[cfg.cache_dtype]
    e = 16 // w
    k = raw[..., :n].contiguous().view(t).to(torch.float64).view(-1, kv, p // 16, d // (4 * e), 4, 16, e)
    v = raw[..., n:2 * n].contiguous().view(t).to(torch.float64).view(-1, kv, p // 16, d // (4 * e), 4, 16, e // 4, 4)
    k = k.permute(0, 1, 2, 5, 3, 4, 6).reshape(-1, kv, p, d)
    v = v.permute(0, 1, 2, 4, 7, 3, 6, 5).reshape(-1, kv, p, d)
    s = raw[..., 2 * n:].contiguous().view(torch.float32).to(torch.float64)
    ks, vs = s[..., :p], s[..., p:]
    return k * ks[..., None], v * vs[..., None], ks, vs


def held(cfg, pool, table, b, end):
    """Keys and values of sequence b, [kv, end, d] float64."""
    k, v, _, _ = natural(cfg, pool)
    pages = torch.as_tensor(np.asarray(table[b])[:-(-end // cfg.page_size)].astype(np.int64))
    return [x[pages].transpose(0, 1).reshape(cfg.n_kv_heads, -1, cfg.head_dim)[:, :end] for x in (k, v)]


def rotate(x, positions, base):
    half = x.shape[-1] // 2
    a = torch.as_tensor(positions, dtype=torch.float64)[:, None] * base ** (-torch.arange(half, dtype=torch.float64) / half)
    c, s = a.cos()[:, None], a.sin()[:, None]
    lo, hi = x[..., :half], x[..., half:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def tables(cfg, ends, seed=0, order=None):
    """A page table that hands out the pool's pages in a random order."""
    order = np.random.RandomState(seed).permutation(cfg.n_pages) if order is None else order
    out, first = [], 0
    for e in ends:
        n = -(-e // cfg.page_size)
        out.append([int(p) for p in order[first:first + n]])
        first += n
    return out


# ------------------------------------------------------------------------------------------ CPU: handle, plan, packers

@pytest.mark.parametrize("over,code", [
    (dict(q=0), B.SPD_EINVAL), (dict(q=6, kv=4), B.SPD_EINVAL), (dict(dtype=B.SPD_F32), B.SPD_EINVAL), (dict(dtype=7), B.SPD_EINVAL),
    (dict(cache=9), B.SPD_EINVAL), (dict(base=0.0), B.SPD_EINVAL), (dict(base=float("nan")), B.SPD_EINVAL), (dict(n_pages=0), B.SPD_EINVAL),
    (dict(max_ctx=0), B.SPD_EINVAL), (dict(d=96), B.SPD_EUNSUPPORTED), (dict(page=48), B.SPD_EUNSUPPORTED),
    (dict(page=512), B.SPD_EUNSUPPORTED), (dict(cache=B.SPD_F16), B.SPD_EUNSUPPORTED), (dict(q=34, kv=2), B.SPD_EUNSUPPORTED)])
def test_pages_create_rejects(over, code):
    with pytest.raises(B.SpdError) as e:
        B.spd_pages_create(config(**over))
    assert e.value.code == code


@pytest.fixture
def pages():
    made = []

    def make(**over):
        cfg = config(**over)
        ctx = B.spd_pages_create(cfg)
        made.append(ctx)
        return cfg, ctx
    yield make
    for ctx in made:
        B.spd_pages_destroy(ctx)


def test_pages_sizes_and_rope(pages):
    cfg, ctx = pages(d=64, page=16, n_pages=3, max_ctx=50, cache=B.SPD_BF16)
    s = B.spd_pages_get_sizes(ctx)
    assert s.pool_bytes == 3 * 2 * 16 * (2 * 64 * 2 + 8) and s.rope_bytes == 50 * 32 * 8
    t = B.spd_pages_rope_table(ctx).reshape(50, 32, 2)
    a = np.arange(50)[:, None] * 10000.0 ** (-np.arange(32) / 32)
    assert np.abs(t[..., 0] - np.cos(a)).max() <= U32 and np.abs(t[..., 1] - np.sin(a)).max() <= U32


@pytest.mark.parametrize("bad", [
    dict(positions=[0], q_lens=[1025]), dict(positions=[-1], q_lens=[1]), dict(positions=[0], q_lens=[-1]),
    dict(table=[[40]]), dict(table=[[-1]]), dict(positions=[31], q_lens=[2]),                          # second page missing
    dict(positions=[0, 0], q_lens=[1, 1], table=[[3], [3]]),                                             # two writers
    dict(positions=[0, 20], q_lens=[1, 0], table=[[3], [3]]),                                            # written and read
    dict(positions=[0], q_lens=[40], table=[[3, 3]]),                                                    # written in two places
    dict(window=-1), dict(sinks=-1, window=4), dict(sinks=2)])
def test_plan_rejects(pages, bad):
    cfg, ctx = pages()
    a = dict(positions=[0], q_lens=[1], table=[[0]], window=0, sinks=0)
    a.update(bad)
    with pytest.raises(B.SpdError) as e:
        B.spd_pages_plan(ctx, a["positions"], a["q_lens"], a["table"], a["window"], a["sinks"])
    assert e.value.code == B.SPD_EINVAL


def test_plan_raw_refusals(pages):
    cfg, ctx = pages()
    lib, n = B.lib(), C.c_size_t()
    one, none = np.array([1], np.int32), np.array([0], np.int32)
    p = lambda a: a.ctypes.data  # noqa: E731
    assert lib.spd_pages_plan(ctx, 1, p(none), p(one), p(none), 1, 0, 0, None, 0, C.byref(n)) == B.SPD_OK and n.value > 0
    buf = np.zeros(n.value, np.uint8)
    assert lib.spd_pages_plan(ctx, 1, p(none), p(one), p(none), 1, 0, 0, p(buf), n.value - 1, C.byref(n)) == B.SPD_EINVAL
    assert lib.spd_pages_plan(ctx, 1, p(none), p(one), p(none), 0, 0, 0, None, 0, C.byref(n)) == B.SPD_EINVAL
    assert lib.spd_pages_plan(None, 1, p(none), p(one), p(none), 1, 0, 0, None, 0, C.byref(n)) == B.SPD_EINVAL
    assert lib.spd_pages_plan(ctx, 1, None, p(one), p(none), 1, 0, 0, None, 0, C.byref(n)) == B.SPD_EINVAL
    assert lib.spd_pages_plan(ctx, -1, p(none), p(one), p(none), 1, 0, 0, None, 0, C.byref(n)) == B.SPD_EINVAL
    assert lib.spd_pages_plan(ctx, 1, p(none), p(one), p(none), 1, 0, 0, None, 0, None) == B.SPD_EINVAL


def test_shared_prefix_is_planned(pages):
    """Pages that nobody writes may be in several sequences."""
    cfg, ctx = pages()
    plan = B.spd_pages_plan(ctx, [64, 70], [1, 3], [[5, 6, 7], [5, 6, 8]])
    i = B.spd_pages_plan_get_info(ctx, plan)
    assert (i.batch, i.tokens, i.held) == (2, 4, 65 + 73)


def test_plan_of_another_pool_is_refused(pages):
    cfg, ctx = pages()
    _, other = pages(page=64)
    plan = B.spd_pages_plan(ctx, [0], [1], [[0]])
    assert B.lib().spd_pages_plan_get_info(other, plan.ctypes.data, C.byref(B.spd_pages_plan_info())) == B.SPD_EINVAL
    assert B.lib().spd_pages_plan_get_info(ctx, np.zeros(4096, np.uint8).ctypes.data, C.byref(B.spd_pages_plan_info())) == B.SPD_EINVAL


def test_empty_plans(pages):
    cfg, ctx = pages()
    for args in (([], [], []), ([0], [0], [[]]), ([5, 0], [0, 0], [[1], []])):
        i = B.spd_pages_plan_get_info(ctx, B.spd_pages_plan(ctx, *args))
        assert i.tokens == 0 and i.workspace_bytes == 0


def test_page_calls_reject_bad_arguments_before_any_launch(pages):
    cfg, ctx = pages()
    plan = B.spd_pages_plan(ctx, [0], [2], [[0]])
    lib, a = B.lib(), np.zeros(4096, np.uint8)
    base = (a.ctypes.data + 255) // 256 * 256
    ph = plan.ctypes.data
    w = (8 + 4) * 128
    write = dict(pages=ctx, ph=ph, pd=base, t=B.SPD_BF16, qkv=base, ld=w, rope=base, pool=base, qo=base + 1024, ldq=1024)
    for over in (dict(pages=None), dict(ph=None), dict(pd=None), dict(pd=base + 4), dict(t=B.SPD_F16), dict(t=B.SPD_E4M3), dict(qkv=None),
                 dict(qkv=base + 2), dict(ld=w - 8), dict(ld=w + 4), dict(pool=None), dict(pool=base + 16), dict(rope=None), dict(ldq=1000),
                 dict(ldq=1028), dict(qo=base + 2), dict(qo=base, ldq=1024), dict(t=B.SPD_F32, qo=base, ldq=w)):
        x = {**write, **over}
        assert lib.spd_pages_write(x["pages"], x["ph"], x["pd"], x["t"], x["qkv"], x["ld"], x["rope"], x["pool"], x["qo"], x["ldq"],
                                   None) == B.SPD_EINVAL, over
    read = dict(pages=ctx, ph=ph, pd=base, pool=base, t=B.SPD_F32, k=base, v=base)
    for over in (dict(pages=None), dict(ph=None), dict(pool=None), dict(t=B.SPD_F16), dict(k=None), dict(v=None), dict(k=base + 4),
                 dict(pool=base + 64)):
        x = {**read, **over}
        assert lib.spd_pages_read(x["pages"], x["ph"], x["pd"], x["pool"], x["t"], x["k"], x["v"], None) == B.SPD_EINVAL, over
    far = base + (1 << 20)
    att = dict(pages=ctx, ph=ph, pd=base, q=base, ldq=1024, pool=base, o=far, ldo=1024)
    for over in (dict(pages=None), dict(ph=None), dict(pd=None), dict(q=None), dict(q=base + 8), dict(ldq=1016), dict(ldq=1028), dict(pool=None),
                 dict(o=None), dict(o=far + 2), dict(ldo=1023), dict(o=base), dict(o=base + 1024)):
        x = {**att, **over}
        assert lib.spd_pages_attention(x["pages"], x["ph"], x["pd"], x["q"], x["ldq"], x["pool"], x["o"], x["ldo"], None, None) == B.SPD_EINVAL, over
    split = B.spd_pages_plan(ctx, [1000], [1], [list(range(32))])          # cut into items: needs its workspace
    assert B.spd_pages_plan_get_info(ctx, split).workspace_bytes > 0
    assert lib.spd_pages_attention(ctx, split.ctypes.data, base, base, 1024, base, far, 1024, None, None) == B.SPD_EINVAL
    assert lib.spd_pages_attention(ctx, split.ctypes.data, base, base, 1024, base, far, 1024, base + 16, None) == B.SPD_EINVAL


def test_rows_and_product_reject_bad_arguments_before_any_launch():
    lib, a = B.lib(), np.zeros(4096, np.uint8)
    base = (a.ctypes.data + 255) // 256 * 256
    norm = dict(t=B.SPD_F32, rows=2, n=8, x=base, ldx=8, add=None, lda=0, g=base, eps=1e-5, s=None, lds=0, c=base, ldc=8, sc=base)
    for over in (dict(t=B.SPD_E4M3), dict(rows=-1), dict(n=-1), dict(x=None), dict(x=base + 2), dict(ldx=7), dict(g=None), dict(eps=-1.0),
                 dict(eps=float("nan")), dict(c=None), dict(ldc=7), dict(sc=None), dict(add=base, lda=7), dict(s=base + 64, lds=4),
                 dict(s=base, lds=16)):
        x = {**norm, **over}
        assert lib.spd_q8_norm(x["t"], x["rows"], x["n"], x["x"], x["ldx"], x["add"], x["lda"], x["g"], x["eps"], x["s"], x["lds"], x["c"],
                               x["ldc"], x["sc"], None) == B.SPD_EINVAL, over
    assert lib.spd_q8_rows(5, 2, 8, base, 8, base, 8, base, None) == B.SPD_EINVAL
    assert lib.spd_q8_swiglu(B.SPD_F32, 2, 8, base, 15, base, 8, base, None) == B.SPD_EINVAL
    assert lib.spd_q8_rows(B.SPD_F32, 0, 8, base, 8, base, 8, base, None) == B.SPD_OK
    mm = dict(rows=2, K=32, N=8, c=base, ldc=32, sc=base, w=base, t=B.SPD_F32, add=None, lda=0, o=base, ldo=8)
    for over in (dict(rows=-1), dict(K=0), dict(K=B.SPD_Q8_MAX_K + 1), dict(N=0), dict(c=None), dict(c=base + 8), dict(ldc=24), dict(ldc=16), dict(sc=None),
                 dict(w=None), dict(w=base + 16), dict(t=B.SPD_E4M3), dict(o=None), dict(o=base + 2), dict(ldo=7), dict(add=base + 1, lda=8),
                 dict(add=base, lda=9), dict(add=base + 64, lda=7)):
        x = {**mm, **over}
        assert lib.spd_q8_matmul(x["rows"], x["K"], x["N"], x["c"], x["ldc"], x["sc"], x["w"], x["t"], x["add"], x["lda"], x["o"], x["ldo"], None,
                                 None) == B.SPD_EINVAL, over
    assert lib.spd_q8_matmul(0, 32, 8, base, 32, base, base, B.SPD_F32, None, 0, base, 8, None, None) == B.SPD_OK


@pytest.mark.parametrize("K,N", [(1, 1), (64, 16), (65, 17), (130, 50)])
def test_q8_packing(K, N):
    r = np.random.RandomState(K)
    codes, scale = r.randint(-127, 128, (K, N)).astype(np.int8), r.rand(N).astype(np.float32)
    packed = B.spd_q8_pack_codes(codes, scale)
    c, s = B.spd_q8_unpack(K, N, packed)
    assert np.array_equal(c, codes) and np.array_equal(s, scale)
    assert packed.size == B.spd_q8_weight_bytes(K, N)
    # every byte that is neither a code nor a scale is zero
    assert np.count_nonzero(packed) <= np.count_nonzero(codes) + 4 * N
    w = r.randn(K, N).astype(np.float32)
    w[:, 0] = 0.0
    c, s = B.spd_q8_unpack(K, N, B.spd_q8_pack(w))
    step = np.maximum(np.abs(w).max(0), LEAST) / 127
    assert np.allclose(s, step, rtol=2.0 ** -23, atol=0)
    assert (np.abs(c * s.astype(np.float64) - w) <= step * (0.5 + 127 * 2.0 ** -22)).all()


def test_q8_pack_rejects():
    w = np.ones((4, 4), np.float32)
    w[2, 1] = np.inf
    with pytest.raises(B.SpdError):
        B.spd_q8_pack(w)
    w = np.ones((4, 4), np.float32)
    out = np.empty(B.spd_q8_weight_bytes(4, 4), np.uint8)
    assert B.lib().spd_q8_pack(4, 4, w.ctypes.data, 3, out.ctypes.data) == B.SPD_EINVAL
    assert B.lib().spd_q8_pack(4, 4, None, 4, out.ctypes.data) == B.SPD_EINVAL
    assert B.spd_q8_weight_bytes(0, 4) == 0 and B.spd_q8_weight_bytes(B.SPD_Q8_MAX_K + 1, 4) == 0


def test_tensors_that_are_not_on_the_device_are_refused(pages):
    cfg, ctx = pages()
    x, codes, scales = torch.zeros(2, 16), torch.zeros(2, 16, dtype=torch.int8), torch.zeros(2)
    B.lib()
    for call in (lambda: B.spd_q8_rows(x, codes, scales), lambda: B.spd_q8_norm(x, None, torch.ones(16), 1e-5, None, codes, scales),
                 lambda: B.spd_q8_swiglu(x, codes[:, :8], scales),
                 lambda: B.spd_q8_matmul(codes, scales, torch.zeros(B.spd_q8_weight_bytes(16, 16), dtype=torch.uint8), 16, None, x)):
        with pytest.raises((ValueError, TypeError)):
            call()


def test_every_workspace_keeps_the_counters_place(pages):
    """Chunks alone, cut into items: the partial results begin behind the counters, which a plan of single tokens shares."""
    cfg, ctx = pages()
    chunk = B.spd_pages_plan_get_info(ctx, B.spd_pages_plan(ctx, [900], [60], [list(range(30))])).workspace_bytes
    rows, heads, d = 128, cfg.n_kv_heads, cfg.head_dim
    assert chunk > 0 and (chunk - 16384 * 4) % (rows * heads * (d + 2) * 4) == 0


# ------------------------------------------------------------------------------------------ GPU: pages

KINDS = [(B.SPD_BF16, B.SPD_E4M3), (B.SPD_F16, B.SPD_E4M3), (B.SPD_BF16, B.SPD_BF16), (B.SPD_F16, B.SPD_F16)]
KIND_IDS = ["bf16-e4m3", "f16-e4m3", "bf16-bf16", "f16-f16"]


class Step:
    """A pool with sequences of given lengths whose first positions were written by an earlier step, and the step's own inputs."""

    def __init__(self, dev, cfg, positions, q_lens, window=0, sinks=0, seed=0, order=None, spoil=None, rope=True, in_f32=False):
        self.cfg, self.positions, self.q_lens = cfg, positions, q_lens
        self.dp = B.DevicePages(cfg, dev)
        self.ends = [p + n for p, n in zip(positions, q_lens)]
        self.table = tables(cfg, self.ends, seed, order)
        g = torch.Generator().manual_seed(seed)
        width = (cfg.n_q_heads + 2 * cfg.n_kv_heads) * cfg.head_dim
        t = T16[cfg.dtype]
        self.rope = self.dp.rope if rope else None
        if sum(positions):         # the positions before the step
            before = B.PagePlan(self.dp, [0] * len(positions), positions, self.table)
            past = torch.randn(sum(positions), width, generator=g).to(t)
            if spoil:
                spoil(self, past)
            B.spd_pages_write(self.dp.ctx, before, past.to(dev), self.rope, self.dp.pool)
        self.plan = B.PagePlan(self.dp, positions, q_lens, self.table, window, sinks)
        self.qkv = torch.randn(sum(q_lens), width, generator=g).to(torch.float32 if in_f32 else t)
        self.qkv_dev = self.qkv.to(dev)
        self.window, self.sinks = window, sinks
        self.q = torch.empty(sum(q_lens), cfg.n_q_heads * cfg.head_dim, dtype=t, device=dev)

    def write(self, q=True):
        B.spd_pages_write(self.dp.ctx, self.plan, self.qkv_dev, self.rope, self.dp.pool, self.q if q and self.rope is not None else None)

    def attend(self, q=None):
        out = torch.full_like(self.q, float("nan"))
        B.spd_pages_attention(self.dp.ctx, self.plan, self.q if q is None else q, self.dp.pool, out, self.plan.workspace)
        return out


def reference(step, q, pool):
    """Attention in 64 bits from the pool's bytes and the queries; and sum of softmax |v| (what a rounded probability moves)."""
    cfg, out, mag, first = step.cfg, [], [], 0
    group, d = cfg.n_q_heads // cfg.n_kv_heads, cfg.head_dim
    for b, (p, n) in enumerate(zip(step.positions, step.q_lens)):
        x = q[first:first + n].double().view(n, cfg.n_q_heads, d)
        first += n
        k, v = held(cfg, pool, step.table, b, p + n)
        at, key = torch.arange(p, p + n)[:, None], torch.arange(p + n)[None]
        seen = key <= at
        if step.window:
            seen &= (key > at - step.window) | (key < step.sinks)
        o, a = torch.zeros(n, cfg.n_q_heads, d, dtype=torch.float64), torch.zeros(n, cfg.n_q_heads, d, dtype=torch.float64)
        for h in range(cfg.n_q_heads):
            s = (x[:, h] @ k[h // group].t()) / math.sqrt(d)
            # hidden keys and values do not count, whatever they hold
            w = torch.where(seen, s, torch.full_like(s, -math.inf)).softmax(-1)
            vv = v[h // group]
            bad = ~torch.isfinite(vv).all(-1)
            clean = torch.where(bad[:, None], torch.zeros_like(vv), vv)
            o[:, h], a[:, h] = w @ clean, w @ clean.abs()
            o[(seen & bad).any(-1), h] = math.nan
        out.append(o.flatten(1))
        mag.append(a.flatten(1))
    return torch.cat(out), torch.cat(mag)


def check_attention(step, got, q=None):
    q = (step.q if q is None else q).cpu()
    want, mag = reference(step, q, step.dp.pool.cpu())
    got = got.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    t = T16[step.cfg.dtype]
    up = U[torch.bfloat16] if step.cfg.cache_dtype == B.SPD_E4M3 else U[t]      # rounding of a probability times its value's scale
    # scores of up to 40 in powers of two: their fp32 rounding moves a probability by 2^-24 * 40 * ln 2 * a few
    bound = (up * 1.01 + 2e-5) * mag + U[t] * want.abs() * 1.01 + 2.0 ** -24
    err = (got - want).abs()
    assert bool((err[~torch.isnan(want)] <= bound[~torch.isnan(want)]).all()), float((err / bound).nan_to_num().max())


LENGTHS = [([0], [1]), ([15], [1]), ([16], [1]), ([700], [1]), ([33, 0, 200, 90], [1, 1, 1, 1]), ([5, 100], [3, 0]), ([0], [17]),
           ([0, 31], [64, 33]), ([130, 7, 0], [70, 1, 129]), ([500], [2]), ([0], [300])]


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("positions,q_lens", LENGTHS, ids=lambda v: "-".join(map(str, v)))
def test_write_then_attend(gpu, dtype, cache, positions, q_lens):
    step = Step(gpu, config(dtype=dtype, cache=cache, page=32, n_pages=60), positions, q_lens, seed=len(positions) + sum(q_lens))
    step.write()
    check_attention(step, step.attend())


@gpu_test
@pytest.mark.parametrize("q,kv,d,page", [(1, 1, 64, 16), (4, 4, 128, 16), (5, 5, 128, 64), (12, 4, 64, 128), (16, 1, 128, 256), (32, 2, 64, 32),
                                         (9, 3, 128, 64)])
@pytest.mark.parametrize("dtype,cache", KINDS[:1] + KINDS[3:], ids=KIND_IDS[:1] + KIND_IDS[3:])
def test_heads_and_pages(gpu, q, kv, d, page, dtype, cache):
    cfg = config(q=q, kv=kv, d=d, page=page, n_pages=3 + 1200 // page, dtype=dtype, cache=cache)
    step = Step(gpu, cfg, [77, 300], [40, 1], seed=q)
    step.write()
    check_attention(step, step.attend())


@gpu_test
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (16, 4), (33, 0), (64, 40), (100, 17), (1000, 4), (5, 600)])
@pytest.mark.parametrize("positions,q_lens", [([200, 3], [1, 1]), ([150], [90]), ([0, 400], [130, 20]), ([320], [3])], ids=str)
def test_window_and_sinks(gpu, window, sinks, positions, q_lens):
    for dtype, cache in (KINDS[0], KINDS[3]):
        step = Step(gpu, config(dtype=dtype, cache=cache, page=16, n_pages=60), positions, q_lens, window=window, sinks=sinks, seed=window)
        step.write()
        check_attention(step, step.attend())


@gpu_test
@pytest.mark.parametrize("dtype,cache", [KINDS[0], KINDS[3]], ids=[KIND_IDS[0], KIND_IDS[3]])
@pytest.mark.parametrize("q_len", [1, 40])
def test_values_that_are_not_finite_reach_only_those_that_see_them(gpu, dtype, cache, q_len):
    cfg = config(dtype=dtype, cache=cache, page=16, n_pages=60)
    width = (cfg.n_q_heads + 2 * cfg.n_kv_heads) * cfg.head_dim
    key0, val0 = cfg.n_q_heads * cfg.head_dim, (cfg.n_q_heads + cfg.n_kv_heads) * cfg.head_dim

    def spoil(step, past):
        past[10, key0 + 3] = math.nan          # hidden from everyone: outside every window, no sink
        past[11, val0 + 5] = math.inf
        past[12, val0 + 200] = -math.inf       # head 1
        past[190, key0 + 7] = math.inf         # visible to the first of the chunk's queries only
        past[191, width - 1] = math.nan        # head 1

    step = Step(gpu, cfg, [200], [q_len], window=12, sinks=4, seed=3, spoil=spoil)
    step.write()
    got = step.attend()
    check_attention(step, got)
    assert torch.isnan(got[0]).any() and (q_len == 1 or not torch.isnan(got[12:]).any())


@gpu_test
def test_pages_that_held_other_sequences(gpu):
    """The rest of a page may hold whatever was there: keys of an earlier sequence, NaN scales among them."""
    cfg = config(page=64, n_pages=4)
    for q_len in (1, 30):
        step = Step(gpu, cfg, [70], [q_len], seed=5)
        dirt = torch.randint(0, 127, step.dp.pool.shape, generator=torch.Generator().manual_seed(1)).to(torch.uint8)
        dirt = torch.where(dirt % 128 == 127, torch.zeros_like(dirt), dirt)
        raw = dirt.view(cfg.n_pages, cfg.n_kv_heads, -1)
        raw[..., 2 * 64 * 128:] = 255                       # every scale NaN
        step.dp.pool.copy_(dirt.view(-1).to(gpu))
        before = B.PagePlan(step.dp, [0], [70], step.table)
        past = torch.randn(70, step.qkv.shape[1]).to(torch.bfloat16).to(gpu)
        B.spd_pages_write(step.dp.ctx, before, past, step.rope, step.dp.pool)
        step.write()
        check_attention(step, step.attend())


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("in_f32", [False, True])
@pytest.mark.parametrize("d,page", [(128, 32), (64, 16)])
def test_write_and_read_back(gpu, dtype, cache, in_f32, d, page):
    cfg = config(dtype=dtype, cache=cache, d=d, page=page, n_pages=80)
    step = Step(gpu, cfg, [0, 37, 100, 15], [50, 1, 20, 2], seed=d, in_f32=in_f32)
    step.qkv[3] = 0.0
    step.qkv[4] *= 1e-30
    step.qkv_dev.copy_(step.qkv)
    untouched = step.dp.pool.clone()
    step.write()
    pool = step.dp.pool.cpu()
    t = T16[dtype]
    nq, nkv, first = cfg.n_q_heads, cfg.n_kv_heads, 0
    new = torch.zeros(cfg.n_pages, cfg.page_size, dtype=torch.bool)
    for b, (p, n) in enumerate(zip(step.positions, step.q_lens)):
        x = step.qkv[first:first + n].double().view(n, nq + 2 * nkv, d)
        at = torch.arange(p, p + n)
        turned = rotate(x, at, cfg.rope_base)
        size = (x[..., :d // 2] ** 2 + x[..., d // 2:] ** 2).sqrt().repeat(1, 1, 2)       # what rounding a rotation scales with
        got = step.q[first:first + n].cpu().double().view(n, nq, d)
        # angles and products in fp32: three roundings of at most the pair's length
        assert bool(((got - turned[:, :nq]).abs() <= U[t] * turned[:, :nq].abs() * 1.01 + 4 * U32 * size[:, :nq] + 2.0 ** -25).all())
        kk, vv = held(cfg, pool, step.table, b, p + n)
        for name, rows, stored in (("key", turned[:, nq:nq + nkv], kk), ("value", x[:, nq + nkv:], vv)):
            rows = rows.transpose(0, 1)
            stored = stored[:, p:]
            noise = 4 * U32 * (size[:, nq:nq + nkv].transpose(0, 1) if name == "key" else rows.abs())
            if cache == B.SPD_E4M3:
                a = rows.abs().amax(-1, keepdim=True).clamp(min=LEAST)
                y = rows * 448 / a
                step_of = 2.0 ** (y.abs().clamp(min=2.0 ** -6).log2().floor() - 3)
                bound = (step_of / 2 * 1.0001 + 448 * 8 * U32) * a / 448 + 2 * noise
            else:
                bound = U[T16[cache]] * rows.abs() * 1.01 + noise + 2.0 ** -25
            assert bool(((stored - rows).abs() <= bound).all()), name
        for i in range(p, p + n):
            new[step.table[b][i // page], i % page] = True
        first += n
    # nothing but the new positions changed
    old, now = natural(cfg, untouched.cpu()), natural(cfg, pool)
    keep = ~new[:, None, :].expand(-1, nkv, -1)
    for o, w in zip(old, now):
        assert torch.equal(o[keep], w[keep])
    # reading back
    for out_t in (torch.float32, t):
        k_out, v_out = (torch.empty(step.plan.info.held, nkv, d, dtype=out_t, device=gpu) for _ in range(2))
        B.spd_pages_read(step.dp.ctx, step.plan, step.dp.pool, k_out, v_out)
        first = 0
        for b, e in enumerate(step.ends):
            for got, want in zip((k_out, v_out), held(cfg, pool, step.table, b, e)):
                got = got[first:first + e].cpu().double().transpose(0, 1)
                # (the smallest fp16 step is 2^-24)
                assert bool(((got - want).abs() <= U[out_t] * want.abs() * 1.0001 + 2.0 ** -25).all())
            first += e


@gpu_test
@pytest.mark.parametrize("dtype,cache", [KINDS[0], KINDS[2], KINDS[3]], ids=[KIND_IDS[0], KIND_IDS[2], KIND_IDS[3]])
def test_rows_that_are_not_finite_are_stored_as_nan(gpu, dtype, cache):
    cfg = config(dtype=dtype, cache=cache)
    step = Step(gpu, cfg, [0], [20], rope=False, in_f32=True)
    k0 = cfg.n_q_heads * cfg.head_dim
    v0 = k0 + cfg.n_kv_heads * cfg.head_dim
    step.qkv[2, k0 + 4] = math.nan
    step.qkv[5, v0 + 1] = math.inf
    step.qkv[7, v0 + 128] = -math.inf
    step.qkv[9, k0 + 100] = 1e6            # past fp16's range
    step.qkv_dev.copy_(step.qkv)
    step.write()
    k, v = held(cfg, step.dp.pool.cpu(), step.table, 0, 20)
    want_k, want_v = torch.zeros(2, 20, dtype=torch.bool), torch.zeros(2, 20, dtype=torch.bool)
    want_k[0, 2] = want_v[0, 5] = want_v[1, 7] = True
    want_k[0, 9] = cache == B.SPD_F16
    for x, want in ((k, want_k), (v, want_v)):
        assert torch.equal(torch.isnan(x).all(-1), want) and torch.equal(torch.isnan(x).any(-1), want)


@gpu_test
def test_queries_in_place_and_strided_rows(gpu):
    """Queries rotated where they stand, attention reading them there and writing into wider rows."""
    cfg = config(q=6, kv=3, d=64, page=16)
    step = Step(gpu, cfg, [20], [37], seed=9)
    plain = torch.empty_like(step.q)
    B.spd_pages_write(step.dp.ctx, step.plan, step.qkv_dev, step.rope, step.dp.pool, plain)
    wide = torch.zeros(37, step.qkv.shape[1] + 16, dtype=torch.bfloat16, device=gpu)
    wide[:, :-16] = step.qkv_dev
    q = wide[:, :6 * 64]
    B.spd_pages_write(step.dp.ctx, step.plan, wide, step.rope, step.dp.pool, q)
    assert torch.equal(q, plain) and torch.equal(wide[:, 6 * 64:-16], step.qkv_dev[:, 6 * 64:])
    out = torch.zeros(37, 500, dtype=torch.bfloat16, device=gpu)[:, :496]
    view = out[:, 56:56 + 6 * 64]
    big = torch.zeros(37, 512, dtype=torch.bfloat16, device=gpu)
    view = big[:, 64:64 + 6 * 64]
    B.spd_pages_attention(step.dp.ctx, step.plan, q, step.dp.pool, view, step.plan.workspace)
    check_attention(step, view, q)
    assert not big[:, :64].any() and not big[:, 64 + 6 * 64:].any()


@gpu_test
def test_pool_beyond_32_bits(gpu):
    """Pages at the end of a pool of more than 4 GiB."""
    cfg = config(q=8, kv=8, d=128, page=256, n_pages=8200, cache=B.SPD_E4M3)
    n = cfg.n_pages
    order = [n - 1, 0, n - 2, 1, n - 3, 4000]
    assert B.spd_pages_get_sizes(B.spd_pages_create(cfg)).pool_bytes > 1 << 32
    step = Step(gpu, cfg, [300, 400], [1, 30], seed=2, order=order)
    step.write()
    out = step.attend().cpu().double()
    used = sorted(order)
    per = step.dp.pool.numel() // n
    small = torch.cat([step.dp.pool[i * per:(i + 1) * per] for i in used]).cpu()
    cfg2 = config(q=8, kv=8, d=128, page=256, n_pages=len(used), cache=B.SPD_E4M3)
    step.cfg, step.table = cfg2, [[used.index(p) for p in row] for row in step.table]
    want, mag = reference(step, step.q.cpu(), small)
    assert bool(((out - want).abs() <= (U[torch.bfloat16] * 1.01 + 2e-5) * mag + U[torch.bfloat16] * want.abs() * 1.01).all())


@gpu_test
def test_shared_prefix(gpu):
    cfg = config(page=16, n_pages=60)
    step = Step(gpu, cfg, [64], [0], seed=4)
    row = step.table[0][:4]
    plan = B.PagePlan(step.dp, [64, 64], [3, 1], [row + [50], row + [51]])
    step.table, step.positions, step.q_lens, step.plan = [row + [50], row + [51]], [64, 64], [3, 1], plan
    step.qkv = torch.randn(4, 12 * 128).to(torch.bfloat16)
    step.qkv_dev = step.qkv.to(gpu)
    step.q = torch.empty(4, 8 * 128, dtype=torch.bfloat16, device=gpu)
    step.write()
    check_attention(step, step.attend())


@gpu_test
def test_step_on_another_stream_in_a_graph_and_twice(gpu):
    """The same bits on another stream, from a graph (several replays, eager work between them) and on a second call."""
    step = Step(gpu, config(page=16, n_pages=120), [700, 64, 0], [1, 80, 3], seed=6)
    step.write()
    want, q = step.attend(), step.q.clone()
    assert torch.equal(step.attend(), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.write()
        other = step.attend()
    side.synchronize()
    assert torch.equal(other, want) and torch.equal(step.q, q)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.spd_pages_write(step.dp.ctx, step.plan, step.qkv_dev, step.rope, step.dp.pool, step.q)
        B.spd_pages_attention(step.dp.ctx, step.plan, step.q, step.dp.pool, out, step.plan.workspace)
    for i in range(3):
        step.q.zero_()
        out.fill_(float(i))
        assert float(out.float().sum()) == out.numel() * i
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(step.attend(), want)


@gpu_test
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("positions,q_lens", [([300, 40], [1, 2]), ([900], [1]), ([200, 0], [70, 40]), ([700], [90])], ids=str)
@pytest.mark.parametrize("values", ["even", "tiny", "mixed"])
def test_fp16_beside_e4m3_rounds_to_fp16(gpu, d, positions, q_lens, values):
    """Probabilities times scales keep fp16's eleven digits, whatever the values' magnitudes."""
    cfg = config(q=8, kv=2, d=d, page=16, n_pages=80, dtype=B.SPD_F16)

    def spoil(step, past):
        n = past.shape[0]
        f = {"even": torch.ones(n), "tiny": torch.full((n,), 3e-4), "mixed": 10.0 ** (torch.arange(n) % 7 - 4.0)}[values]
        past[:, 10 * d:] *= f[:, None].to(past.dtype)
    step = Step(gpu, cfg, positions, q_lens, seed=4, spoil=spoil)
    if values == "tiny":
        step.qkv[:, 10 * d:] *= 3e-4
        step.qkv_dev = step.qkv.to(gpu)
    step.write()
    got, pool = step.attend().cpu().double(), step.dp.pool.cpu()
    want, mag = reference(step, step.q.cpu(), pool)
    # a weight below fp16's normal numbers is off by 2^-25 of the largest weight, which stands for the largest probability times its scale;
    # times codes of up to 448, over all keys
    floor, first = torch.zeros_like(want), 0
    for b, (p, n) in enumerate(zip(positions, q_lens)):
        k, v = held(cfg, pool, step.table, b, p + n)
        x = step.q.cpu()[first:first + n].double().view(n, 8, d)
        hidden = torch.arange(p + n)[None] > torch.arange(p, p + n)[:, None]
        for h in range(8):
            w = (x[:, h] @ k[h // 4].t() / math.sqrt(d)).masked_fill(hidden, -math.inf).softmax(-1)
            most = (w * v[h // 4].abs().amax(-1)).amax(-1)
            floor[first:first + n, h * d:(h + 1) * d] = ((p + n) * 2.0 ** -25 * most)[:, None]
        first += n
    t = torch.float16
    bound = (U[t] * 1.01 + 2e-5) * mag + U[t] * want.abs() * 1.01 + 2.0 ** -25 + floor
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())


@gpu_test
def test_one_workspace_for_several_plans(gpu):
    cfg = config(page=16, n_pages=200)
    steps = [Step(gpu, cfg, p, n, seed=9) for p, n in (([900], [60]), ([1000], [1]), ([640, 900], [33, 1]))]
    wants = []
    for step in steps:
        step.write()
        wants.append(step.attend())
    shared = torch.zeros(max(s.plan.workspace_bytes for s in steps), dtype=torch.uint8, device=gpu)
    for i in (0, 1, 2, 1, 0, 2, 1):
        step, out = steps[i], torch.full_like(wants[i], float("nan"))
        B.spd_pages_attention(step.dp.ctx, step.plan, step.q, step.dp.pool, out, shared)
        assert torch.equal(out, wants[i])


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("up", [True, False])
def test_scores_that_rise_and_fall_along_the_keys(gpu, dtype, cache, up):
    """Maxima that grow by far more than a tile's room, or not at all after the first tile."""
    cfg = config(q=4, kv=2, page=16, n_pages=60, dtype=dtype, cache=cache)

    def spoil(step, past):
        n = past.shape[0]
        k = past[:, 4 * 128:6 * 128]
        k *= torch.linspace(0.1, 8.0, n).flip(0 if not up else []).to(past.dtype)[:, None]
    step = Step(gpu, cfg, [400, 390], [90, 1], seed=3, spoil=spoil)
    step.write()
    q = (step.q.float() * 4).to(step.q.dtype)
    got = step.attend(q).cpu().double()
    want, mag = reference(step, q.cpu(), step.dp.pool.cpu())
    # scores of up to s in units of e: sums of 128 products in fp32 (at most 16 of them one after the other) and three factors move them by
    # 20 u s, and a probability by as much
    k = torch.cat([held(cfg, step.dp.pool.cpu(), step.table, b, step.ends[b])[0].flatten(0, 1) for b in range(2)])
    s = float(q.float().cpu().view(-1, 128).norm(dim=-1).max() * k.norm(dim=-1).max()) / math.sqrt(128)
    t = T16[dtype]
    rounded = U[torch.bfloat16] if cache == B.SPD_E4M3 else U[t]
    bound = (rounded * 1.01 + 2 * 20 * U32 * s + 2e-5) * mag + U[t] * want.abs() * 1.01 + 2.0 ** -24
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())


@gpu_test
def test_empty_steps(gpu):
    cfg = config()
    dp = B.DevicePages(cfg, gpu)
    for args in (([], [], []), ([3, 0], [0, 0], [[1], []])):
        plan = B.PagePlan(dp, *args)
        x = torch.empty(0, 12 * 128, dtype=torch.bfloat16, device=gpu)
        assert plan.info.tokens == 0
        some = torch.zeros(1, 12 * 128, dtype=torch.bfloat16, device=gpu)
        lib = B.lib()
        p = plan.device.data_ptr()
        assert lib.spd_pages_write(dp.ctx, plan.host.ctypes.data, p, B.SPD_BF16, some.data_ptr(), 1536, None, dp.pool.data_ptr(), None, 0,
                                   None) == B.SPD_OK
        assert lib.spd_pages_attention(dp.ctx, plan.host.ctypes.data, p, some.data_ptr(), 1024, dp.pool.data_ptr(),
                                       some.data_ptr(), 1024, None, None) == B.SPD_OK
        del x


# ------------------------------------------------------------------------------------------ GPU: rows

def check_rows(codes, scales, v, noise):
    """codes * scales against the exact values v: half a step, and `noise` (relative) of what is computed before it."""
    a = v.abs().amax(-1, keepdim=True).clamp(min=LEAST)
    got = codes.cpu().double() * scales.cpu().double()[:, None]
    assert bool((codes.cpu().abs() <= 127).all())
    assert bool(((scales.cpu().double()[:, None] * 127 - a).abs() <= a * (noise + 4 * U32)).all())
    assert bool(((got - v).abs() <= a * (0.5 / 127 + 2 * noise + 8 * U32)).all())


ROWS = [(1, 1), (1, 8192), (3, 7), (16, 8192), (5, 5120), (2, 9001), (300, 688), (4, 16384), (2, 20000), (7, 257), (2, 40001)]


@gpu_test
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n", ROWS)
@pytest.mark.parametrize("add", [False, True])
def test_norm(gpu, t, rows, n, add):
    t = TYPES[t]
    g = torch.Generator().manual_seed(rows * 31 + n)
    x, y = (torch.randn(rows, n, generator=g).to(t) for _ in range(2))
    gain = 1 + 0.1 * torch.randn(n, generator=g)
    codes, scales = torch.empty(rows, n, dtype=torch.int8, device=gpu), torch.empty(rows, device=gpu)
    total = torch.empty(rows, n, dtype=t, device=gpu)
    B.spd_q8_norm(x.to(gpu), y.to(gpu) if add else None, gain.to(gpu), 1e-5, total if add else None, codes, scales)
    s = x.double() + (y.double() if add else 0)
    v = s / (s.square().mean(-1, keepdim=True) + 1e-5).sqrt() * gain.double()
    # a sum of n squares, at most n / 256 of them one after the other and ten levels of partial sums
    noise = (n / 256 + 20) * U32
    check_rows(codes, scales, v, noise + 6 * U32)
    if add:
        assert bool(((total.cpu().double() - s).abs() <= U[t] * s.abs() * 1.0001 + 2.0 ** -25).all())


@gpu_test
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,n", ROWS)
def test_rows_and_swiglu(gpu, t, rows, n):
    t = TYPES[t]
    g = torch.Generator().manual_seed(rows * 17 + n)
    x = (3 * torch.randn(rows, 2 * n, generator=g)).to(t)
    codes, scales = torch.empty(rows, n, dtype=torch.int8, device=gpu), torch.empty(rows, device=gpu)
    B.spd_q8_rows(x[:, :n].to(gpu), codes, scales)
    check_rows(codes, scales, x[:, :n].double(), 0.0)
    B.spd_q8_swiglu(x.to(gpu), codes, scales)
    gate, up = x.double().chunk(2, -1)
    # exp, a sum, a quotient and a product in fp32; exp's argument to 20 in 24 bits
    check_rows(codes, scales, gate * torch.sigmoid(gate) * up, 40 * U32)


@gpu_test
def test_rows_strides_aliases_and_edges(gpu):
    g = torch.Generator().manual_seed(1)
    wide = torch.randn(6, 70, generator=g).to(gpu)
    x, add = wide[:, 1:34], torch.randn(6, 50, generator=g).to(gpu)[:, 3:36]
    gain = torch.ones(33, device=gpu)
    codes = torch.full((6, 48), 99, dtype=torch.int8, device=gpu)
    scales = torch.empty(6, device=gpu)
    s = (x + add).cpu().double()
    before = wide.clone()
    B.spd_q8_norm(x, add, gain, 0.0, x, codes[:, :33], scales)       # the sum in place of the first summand
    assert torch.equal(x.cpu(), s.float()) and torch.equal(wide[:, 34:], before[:, 34:]) and torch.equal(wide[:, 0], before[:, 0])
    assert bool((codes[:, 33:] == 99).all())
    check_rows(codes[:, :33], scales, s / s.square().mean(-1, keepdim=True).sqrt(), 30 * U32)
    # rows of zeros, of tiny and of huge values, and rows that are not finite
    x = torch.randn(9, 64, generator=g)
    x[0], x[1] = 0.0, x[1] * 1e-38
    x[2] *= 1e18
    x[3, 5], x[4, 63], x[5, 0] = math.nan, math.inf, -math.inf
    codes, scales = torch.empty(9, 64, dtype=torch.int8, device=gpu), torch.empty(9, device=gpu)
    bad = torch.zeros(9, dtype=torch.bool)
    bad[3:6] = True
    B.spd_q8_rows(x.to(gpu), codes, scales)
    assert torch.equal(torch.isnan(scales.cpu()), bad)
    check_rows(codes[~bad.to(gpu)], scales[~bad.to(gpu)], x[~bad].double(), 0.0)
    B.spd_q8_norm(x.to(gpu), None, torch.ones(64, device=gpu), 1e-5, None, codes, scales)
    assert torch.equal(torch.isnan(scales.cpu()), bad)
    assert not codes[0].any()
    B.spd_q8_norm(x.to(gpu), None, torch.ones(64, device=gpu), 0.0, None, codes, scales)      # 0 / 0
    assert bool(torch.isnan(scales[0])) and not codes[0].any()
    B.spd_q8_swiglu(torch.cat([x, x], 1).to(gpu), codes, scales)
    assert torch.isnan(scales.cpu())[3:5].all() and not torch.isnan(scales.cpu())[:2].any()


# ------------------------------------------------------------------------------------------ GPU: product

def product(dev, rows, K, N, t, add=False, seed=0, pad=0, full=False):
    g = torch.Generator().manual_seed(seed + rows + K + N)
    ld = (K + 15) // 16 * 16 + pad
    a = torch.randint(-127, 128, (rows, ld), generator=g).to(torch.int8)
    w = torch.randint(-127, 128, (K, N), generator=g).to(torch.int8)
    if full:                       # the largest sums there are
        a[:], w[:] = 127, 127
    sa, sw = torch.rand(rows, generator=g) + 0.01, torch.rand(N, generator=g) + 0.01
    y = torch.randn(rows, N, generator=g).to(t) * 1000 if add else None
    packed = torch.from_numpy(B.spd_q8_pack_codes(w.numpy(), sw.numpy())).to(dev)
    out = torch.full((rows, N + 3), 5.0, dtype=t, device=dev)
    n = B.spd_q8_matmul_workspace(rows, K, N)
    ws = torch.empty(n, dtype=torch.uint8, device=dev) if n else None
    B.spd_q8_matmul(a.to(dev)[:, :K], sa.to(dev), packed, N, y.to(dev) if add else None, out[:, :N], ws)
    p = (a[:, :K].double() @ w.double()) * sa.double()[:, None] * sw.double()
    want = p + (y.double() if add else 0)
    got = out.cpu().double()
    assert bool((got[:, N:] == 5.0).all())
    got = got[:, :N]
    big = torch.finfo(t).max
    fits = want.abs() < big
    bound = 4 * U32 * p.abs() + 2 * U32 * want.abs() + U[t] * want.abs() * 1.0001 + 2.0 ** -25
    assert bool(((got - want).abs() <= bound)[fits].all()), float(((got - want).abs() / bound)[fits].max())
    return out


PRODUCTS = [(1, 1, 1), (1, 64, 16), (1, 8192, 1280), (2, 100, 33), (16, 8192, 7168), (17, 256, 688), (15, 640, 5120), (33, 1376, 257), (64, 4096, 1536),
            (65, 512, 4096), (128, 1024, 8192), (129, 1728, 500), (333, 1728, 5120), (500, 3584, 8192), (700, 130, 1000), (1000, 8192, 1280),
            (257, 64, 300), (2100, 192, 1027), (48, 20000, 64)]


@gpu_test
@pytest.mark.parametrize("rows,K,N", PRODUCTS)
def test_product(gpu, rows, K, N):
    for i, t in enumerate(TYPES.values()):
        product(gpu, rows, K, N, t, add=(rows + i) % 2 == 0, pad=16 * (i == 1))


@gpu_test
@pytest.mark.parametrize("rows,N", [(3, 17), (200, 40)])
def test_product_of_the_longest_contraction(gpu, rows, N):
    product(gpu, rows, B.SPD_Q8_MAX_K, N, torch.float32, full=True)


@gpu_test
@pytest.mark.parametrize("rows,K,N,t,add", [(2100, 7201, 4100, "f32", False), (4500, 7232, 4104, "bf16", True), (2050, 7168, 4111, "f16", False)])
def test_product_of_many_rows_and_a_long_contraction(gpu, rows, K, N, t, add):
    t, g = TYPES[t], torch.Generator(device=gpu).manual_seed(rows)
    a = torch.randint(-127, 128, (rows, (K + 15) // 16 * 16), generator=g, device=gpu).to(torch.int8)
    w = torch.randint(-127, 128, (K, N), generator=g, device=gpu).to(torch.int8)
    sa, sw = 0.01 + torch.rand(rows, generator=g, device=gpu), 1e-3 * (0.01 + torch.rand(N, generator=g, device=gpu))
    y = torch.randn(rows, N, generator=g, device=gpu).to(t) * 100 if add else None
    packed = torch.from_numpy(B.spd_q8_pack_codes(w.cpu().numpy(), sw.cpu().numpy())).to(gpu)
    out = torch.empty(rows, N, dtype=t, device=gpu)
    B.spd_q8_matmul(a[:, :K], sa, packed, N, y, out)
    p = (a[:, :K].double() @ w.double()) * sa.double()[:, None] * sw.double()      # (whole numbers far below 2^53: exact)
    want = p + (y.double() if add else 0)
    bound = 4 * U32 * p.abs() + 2 * U32 * want.abs() + U[t] * want.abs() * 1.0001 + 2.0 ** -25
    fits = want.abs() < torch.finfo(t).max
    assert bool(((out.double() - want).abs() <= bound)[fits].all())


@gpu_test
def test_product_adds_in_place_and_keeps_its_bits(gpu):
    for rows in (5, 40, 300, 1000):
        K, N = 700, 530
        g = torch.Generator().manual_seed(rows)
        a = torch.randint(-127, 128, (rows, 704), generator=g).to(torch.int8).to(gpu)[:, :K]
        w = torch.randint(-127, 128, (K, N), generator=g).to(torch.int8)
        sa, sw = torch.rand(rows, generator=g).to(gpu), torch.rand(N, generator=g)
        packed = torch.from_numpy(B.spd_q8_pack_codes(w.numpy(), sw.numpy())).to(gpu)
        y = torch.randn(rows, N, generator=g).to(gpu)
        n = B.spd_q8_matmul_workspace(rows, K, N)
        ws = torch.empty(n, dtype=torch.uint8, device=gpu) if n else None
        out, again = torch.empty(rows, N, device=gpu), y.clone()
        B.spd_q8_matmul(a, sa, packed, N, y, out, ws)
        B.spd_q8_matmul(a, sa, packed, N, again, again, ws)
        assert torch.equal(out, again)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        third = torch.empty_like(out)
        B.spd_q8_matmul(a, sa, packed, N, y, third, ws, stream=stream)
        stream.synchronize()
        assert torch.equal(out, third)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.spd_q8_matmul(a, sa, packed, N, y, third, ws)
        for i in range(3):
            third.fill_(i)
            assert float(third.sum()) == third.numel() * i
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, third)


# ------------------------------------------------------------------------------------------ GPU: all of them together

def _example():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "paged_q8_block.py")
    spec = importlib.util.spec_from_file_location("paged_q8_block", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@gpu_test
@pytest.mark.parametrize("cache", [B.SPD_E4M3, B.SPD_BF16], ids=["e4m3", "bf16"])
def test_block_in_8_bits_over_pages(gpu, cache):
    """An SPD block of one rank: chunks of a prompt beside decode steps, against the same block in 64 bits with nothing rounded.

    Per projection: an operand whose largest value is 4 to 5 times its rms is rounded in steps of that over 127, an error of 4.5 / 127 / sqrt(12) = 1 % of its
    rms, for rows and weights 1.5 % of the product; e4m3 rounds keys and values by 2^-4 / sqrt(3) = 3.6 % at most.  Scores of about unit size
    turn the error of queries and keys into as much of the probabilities.  QKV, cache, attention, O: sqrt(1.5^2 (3 times) + 3.6^2 (twice) +
    1 + ...) below 7 %; the MLP on it below 8 %."""
    from paper_2502_20727_amd import inputs, workloads
    ex = _example()
    w = workloads.Workload(name="q8-block", hidden=512, n_q_heads=16, n_kv_heads=4, head_dim=64, ffn=1376, n_layers=1, tp=2, dtype=workloads.BF16,
                           seed=11, batch=3, q_len=1, ctx=64, mask=(1,))
    rank = 1
    shard = inputs.layer_shard(w, 0, rank)
    block = ex.Q8Block(w, shard, rank, max_tokens=200, n_pages=40, page_size=16, max_ctx=512, cache=cache)
    pool = ex.PagedPool(40, 16)
    W = {n: torch.from_numpy(a).double() for n, a in shard.items()}
    q, kv, d = w.q_per_rank, w.kv_per_rank, w.head_dim
    past = [[torch.zeros(0, kv, d, dtype=torch.float64) for _ in range(2)] for _ in range(3)]
    g = torch.Generator().manual_seed(0)
    done = [0, 0, 0]

    def norm(t, gain):
        return t / (t.square().mean(-1, keepdim=True) + w.rms_eps).sqrt() * gain

    for lens in ([40, 0, 3], [1, 90, 1], [1, 60, 1], [1, 1, 1], [1, 1, 0]):
        for s, n in enumerate(lens):
            pool.grow(s, done[s] + n)
        plan = B.PagePlan(block.pages, done, lens, [pool.table.get(s, []) for s in range(3)], window=100, sinks=4)
        x = torch.randn(sum(lens), w.hidden, generator=g)
        slots = 0.05 * torch.randn(w.tp, sum(lens), w.hidden, generator=g)
        xd, sd = x.to(gpu), slots.to(gpu)
        out = torch.empty_like(xd)
        block.forward(plan, xd, sd, out)
        X = x.double()
        qkv = norm(X, W["g1"])
        Q, K, V = ((qkv @ W[n]).unflatten(-1, (-1, d)) for n in ("wq", "wk", "wv"))
        att, first = [], 0
        for s, n in enumerate(lens):
            at = torch.arange(done[s], done[s] + n)
            rows = slice(first, first + n)
            first += n
            past[s][0] = torch.cat([past[s][0], rotate(K[rows], at, w.rope_base)])
            past[s][1] = torch.cat([past[s][1], V[rows]])
            key = torch.arange(done[s] + n)
            seen = (key <= at[:, None]) & ((key > at[:, None] - 100) | (key < 4))
            qs, o = rotate(Q[rows], at, w.rope_base), torch.zeros(n, q, d, dtype=torch.float64)
            for j in range(q):
                sc = qs[:, j] @ past[s][0][:, j // (q // kv)].t() / math.sqrt(d)
                o[:, j] = sc.masked_fill(~seen, -math.inf).softmax(-1) @ past[s][1][:, j // (q // kv)]
            att.append(o.flatten(1))
            done[s] += n
        y = torch.cat(att) @ W["wo"]
        m = norm(X + y, W["g2"])
        gate = m @ W["wg"]
        z = (gate * torch.sigmoid(gate) * (m @ W["wu"])) @ W["wd"]
        got = sd[rank].cpu().double()
        assert float((got - (y + z)).norm() / (y + z).norm()) < 0.08
        total = X + slots[0].double() + got
        assert float((out.cpu().double() - total).abs().max()) < 1e-5
    block.close()
