"""Pages in 4 bits (cache_dtype SPD_E2M1 of include/spd_q8.h): refusals on the CPU, numerics on the GPU against plain computations in 64 bits.

What a pool holds is compared exactly: the codes are defined by values in 64 bits, and code * scale is a value of the 16-bit type.
Tolerances elsewhere count roundings: u = torch.finfo(t).eps / 2 of a value rounded to type t."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2502_20727_amd import binding as B
from tests.test_q8_serving import LENGTHS, T16, U, U32, Step, config as config8

gpu_test = pytest.mark.gpu
TYPES = [B.SPD_BF16, B.SPD_F16]
TYPE_IDS = ["bf16", "f16"]
EXPONENTS = {B.SPD_BF16: (-100, 125), B.SPD_F16: (-23, 13)}
SIZES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def config(**over):
    return config8(**{"cache": B.SPD_E2M1, **over})


def quantised(x, dtype):
    """Rows x [..., d] in 64 bits -> what 4 bits make of them: values (NaN for rows that are not finite in the type), exponents [..., d / 32]."""
    lo, hi = EXPONENTS[dtype]
    bad = ~torch.isfinite(x.to(T16[dtype])).all(-1)
    g = torch.where(bad[..., None], torch.zeros_like(x), x).unflatten(-1, (-1, 32))
    a = g.abs().amax(-1)
    e = torch.full_like(a, hi)
    for i in range(hi - 1, lo - 1, -1):            # the least that will do
        e = torch.where(a <= 7 * 2.0 ** i, i, e)
    y = g.abs() / 2.0 ** e[..., None]
    # the nearest of the sizes, of two as near the one of even number
    far = (y[..., None] - SIZES.to(y.device)).abs()
    near = far == far.amin(-1, keepdim=True)
    number = torch.arange(8, device=y.device)
    code = torch.where(near, number % 2 * 8 + number, 99).amin(-1) % 8
    v = (SIZES.to(y.device)[code] * torch.sign(g) * 2.0 ** e[..., None]).flatten(-2)
    return torch.where(bad[..., None], math.nan, v), torch.where(bad[..., None], 128, e)


def natural(cfg, pool):
    """(keys, values) of a pool (bytes, CPU) as [pages, kv, position, d] float64; and the exponents [pages, kv, position, d / 32] (128: NaN)."""
    p, d, kv = cfg.page_size, cfg.head_dim, cfg.n_kv_heads
    n, m = p * d // 2, p * d // 32
    raw = pool.view(cfg.n_pages, kv, 2 * n + 2 * m)
    out, exps = [], []
    signed = torch.cat([SIZES, -SIZES])
    for i in range(2):
        b = raw[..., i * n:(i + 1) * n].contiguous().long()
        both = torch.stack([signed[b & 15], signed[b >> 4]], -1)
        if i == 0:        # [block][g][position][bytes of consecutive features]
            x = both.view(-1, kv, p // 16, 4, 16, d // 8, 2).permute(0, 1, 2, 4, 3, 5, 6)
        else:             # [block][g][r][u][position of four], features r + 32 u and 16 behind it
            x = both.view(-1, kv, p // 16, 4, 16, d // 32, 4, 2).permute(0, 1, 2, 3, 6, 5, 7, 4)
        e = raw[..., 2 * n + i * m:2 * n + (i + 1) * m].contiguous().view(-1, kv, p, d // 32).double() - 127
        x = x.reshape(-1, kv, p, d // 32, 32) * torch.where(e == 128, math.nan, 2.0 ** e)[..., None]
        out.append(x.flatten(-2))
        exps.append(e)
    return out[0], out[1], exps[0], exps[1]


def held(cfg, pool, table, b, end):
    """Keys and values of sequence b, [kv, end, d] float64."""
    pages = torch.as_tensor(np.asarray(table[b])[:-(-end // cfg.page_size)].astype(np.int64))
    per = pool.numel() // cfg.n_pages
    few = pool.view(cfg.n_pages, per)[pages].contiguous()
    small = B.spd_pages_config(cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.page_size, len(pages), cfg.dtype, cfg.cache_dtype, cfg.max_ctx, cfg.rope_base)
    k, v, _, _ = natural(small, few.view(-1))
    return [x.transpose(0, 1).reshape(cfg.n_kv_heads, -1, cfg.head_dim)[:, :end] for x in (k, v)]


def rotate(x, table):
    """x [tokens, heads, d] by cos, sin [tokens, d / 2, 2] in 64 bits."""
    c, s = (t[:, None] for t in table.double().unbind(-1))
    lo, hi = x.chunk(2, -1)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1)


def check_attention(step, got, q=None):
    """As close as the pool's type allows: a probability is rounded to it once (below fp16's normal numbers by 2^-25 of the largest), the output once;
    2e-5: what the scores' rounding in 32 bits moves a probability by."""
    q = (step.q if q is None else q).cpu()
    cfg, pool, t, first = step.cfg, step.dp.pool.cpu(), T16[step.cfg.dtype], 0
    group, d, got = cfg.n_q_heads // cfg.n_kv_heads, cfg.head_dim, got.cpu().double()
    for b, (p, n) in enumerate(zip(step.positions, step.q_lens)):
        if not n:
            continue
        x = q[first:first + n].double().view(n, cfg.n_kv_heads, group, d)
        mine = got[first:first + n].view(n, cfg.n_kv_heads, group, d)
        first += n
        k, v = held(cfg, pool, step.table, b, p + n)
        at, key = torch.arange(p, p + n)[:, None], torch.arange(p + n)[None]
        seen = key <= at
        if step.window:
            seen &= (key > at - step.window) | (key < step.sinks)
        for h in range(cfg.n_kv_heads):
            bad = ~(torch.isfinite(k[h]).all(-1) & torch.isfinite(v[h]).all(-1))
            kk, vv = (torch.where(bad[:, None], 0.0, z[h]) for z in (k, v))
            w = torch.where(seen[:, None], x[:, h] @ kk.t() / math.sqrt(d), -math.inf).softmax(-1)        # [n, group, keys]
            want, mag, none = w @ vv, w @ vv.abs(), (seen & bad).any(-1)
            assert torch.equal(torch.isnan(mine[:, h]), none[:, None, None].expand_as(want))
            floor = 0.0 if t is torch.bfloat16 else (p + n) * 2.0 ** -25 * w.amax(-1, keepdim=True) * vv.abs().max()
            bound = (U[t] * 1.01 + 2e-5) * mag + U[t] * want.abs() * 1.01 + 2.0 ** -24 + floor
            err = (mine[:, h] - want).abs()
            assert bool((err <= bound)[~none].all()), (b, h, float((err / bound)[~none].max()))


# ------------------------------------------------------------------------------------------ CPU

def test_sizes_and_refusals():
    ctx = B.spd_pages_create(config(q=8, kv=2, d=128, page=32, n_pages=7))
    assert B.spd_pages_get_sizes(ctx).pool_bytes == 7 * 2 * 32 * (2 * 64 + 2 * 4)
    B.spd_pages_destroy(ctx)
    ctx = B.spd_pages_create(config(q=8, kv=2, d=64, page=16, n_pages=7, dtype=B.SPD_F16))
    assert B.spd_pages_get_sizes(ctx).pool_bytes == 7 * 2 * 16 * (2 * 32 + 2 * 2)
    B.spd_pages_destroy(ctx)
    for over, code in ((dict(dtype=B.SPD_E2M1), B.SPD_EINVAL), (dict(dtype=B.SPD_F32), B.SPD_EINVAL), (dict(cache=5), B.SPD_EINVAL), (dict(d=32), B.SPD_EUNSUPPORTED),
                       (dict(page=8), B.SPD_EUNSUPPORTED), (dict(q=34, kv=2), B.SPD_EUNSUPPORTED)):
        with pytest.raises(B.SpdError) as e:
            B.spd_pages_create(config(**over))
        assert e.value.code == code


def test_a_pool_of_another_kind_does_not_take_the_plan():
    four, eight = B.spd_pages_create(config()), B.spd_pages_create(config8())
    plan = B.spd_pages_plan(eight, [0], [4], [[1]])
    with pytest.raises(B.SpdError) as e:
        B.spd_pages_plan_get_info(four, plan)
    assert e.value.code == B.SPD_EINVAL
    for p in (four, eight):
        B.spd_pages_destroy(p)


def test_calls_refuse_what_they_cannot_work_on():
    """Host checks alone: nothing is enqueued."""
    cfg = config(q=8, kv=2, d=128, page=32)
    ctx, l = B.spd_pages_create(cfg), B.lib()
    plan = B.spd_pages_plan(ctx, [0], [4], [[1]])
    base = 1 << 20
    wr = lambda t=B.SPD_BF16, qkv=base, ld=12 * 128, rope=base, pool=base, q=base * 2, ldq=1024: l.spd_pages_write(      # noqa: E731
        ctx, plan.ctypes.data, base, t, qkv, ld, rope, pool, q, ldq, None)
    for over in (dict(t=B.SPD_F16), dict(t=B.SPD_E2M1), dict(qkv=base + 2), dict(qkv=None), dict(ld=1535), dict(ld=1537), dict(pool=base + 128), dict(pool=None), dict(rope=None),
                 dict(rope=base + 4), dict(q=base + 64), dict(ldq=1023), dict(ldq=1028), dict(q=base, ldq=1024)):
        assert wr(**over) == B.SPD_EINVAL, over
    rd = lambda pool=base, t=B.SPD_BF16, k=base, v=base: l.spd_pages_read(ctx, plan.ctypes.data, base, pool, t, k, v, None)      # noqa: E731
    for over in (dict(t=B.SPD_E2M1), dict(t=B.SPD_F16), dict(pool=None), dict(k=None), dict(v=base + 8), dict(pool=base + 16)):
        assert rd(**over) == B.SPD_EINVAL, over
    at = lambda q=base, ldq=1024, pool=base, o=base * 2, ldo=1024: l.spd_pages_attention(ctx, plan.ctypes.data, base, q, ldq, pool, o, ldo, None, None)   # noqa: E731
    for over in (dict(q=None), dict(q=base + 2), dict(ldq=1000), dict(ldo=1020), dict(pool=base + 32), dict(o=None), dict(o=base), dict(o=base + 2048)):
        assert at(**over) == B.SPD_EINVAL, over
    B.spd_pages_destroy(ctx)


def test_the_plain_quantiser_itself():
    """The test's own: borders, ties, ends of the range."""
    x = torch.zeros(1, 32, dtype=torch.float64)
    x[0, :14] = torch.tensor([6.0, 7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0001, 0.2500001, -0.25, 6.9, 4.9])
    v, e = quantised(x, B.SPD_BF16)
    assert e[0, 0] == 0 and v[0, :14].tolist() == [6, 6, 0, 1, 1, 2, 2, 4, 4, -6, 0.5, 0, 6, 4]
    x[0, 1] = 7.0000001
    assert quantised(x, B.SPD_BF16)[1][0, 0] == 1
    assert quantised(x * 0, B.SPD_BF16)[1][0, 0] == -100 and quantised(x * 0, B.SPD_F16)[1][0, 0] == -23
    assert quantised(x * 9000, B.SPD_F16)[0][0, 1] == 6 * 2.0 ** 13 and torch.isnan(quantised(x * 9360, B.SPD_F16)[0]).all()


# ------------------------------------------------------------------------------------------ GPU: writing and reading back

@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("in_f32", [False, True])
@pytest.mark.parametrize("q,kv,d,page", [(8, 2, 128, 32), (4, 4, 64, 16), (5, 5, 128, 64), (16, 1, 64, 256), (9, 3, 64, 128)])
def test_write_and_read_back(gpu, dtype, in_f32, q, kv, d, page):
    cfg = config(dtype=dtype, q=q, kv=kv, d=d, page=page, n_pages=80)
    step = Step(gpu, cfg, [0, 37, 100, 15, 48], [50, 1, 20, 2, 16], seed=d + kv, in_f32=in_f32)
    step.qkv[3] = 0.0
    step.qkv[4] *= 2.0 ** -20
    step.qkv[5] *= 100.0
    step.qkv_dev.copy_(step.qkv)
    before = step.dp.pool.cpu()
    step.write()
    pool, rope = step.dp.pool.cpu(), step.rope.cpu().view(-1, d // 2, 2)
    want, first = list(natural(cfg, before)), 0
    for b, (p, n) in enumerate(zip(step.positions, step.q_lens)):
        x = step.qkv[first:first + n].double().view(n, q + 2 * kv, d)
        at = torch.arange(p, p + n)
        turned = rotate(x, rope[at])
        size = (x[..., :d // 2] ** 2 + x[..., d // 2:] ** 2).sqrt().repeat(1, 1, 2)
        got = step.q[first:first + n].cpu().double().view(n, q, d)
        # queries in fp32: three roundings of at most the pair's length
        assert bool(((got - turned[:, :q]).abs() <= U[T16[dtype]] * turned[:, :q].abs() * 1.01 + 4 * U32 * size[:, :q] + 2.0 ** -25).all())
        first += n
        page_of = torch.tensor(step.table[b])[at // page]
        for i, rows in enumerate((turned[:, q:q + kv], x[:, q + kv:])):
            v, e = quantised(rows, dtype)
            want[i][page_of, :, at % page], want[2 + i][page_of, :, at % page] = v, e
    # every code and exponent, the new positions' and those that nothing was written to
    for w, g in zip(want, natural(cfg, pool)):
        assert torch.equal(w, g)
    for out_t in (torch.float32, T16[dtype]):
        k_out, v_out = (torch.full((step.plan.info.held, kv, d), math.nan, dtype=out_t, device=gpu) for _ in range(2))
        B.spd_pages_read(step.dp.ctx, step.plan, step.dp.pool, k_out, v_out)
        first = 0
        for b, e in enumerate(step.ends):
            for g, w in zip((k_out, v_out), held(cfg, pool, step.table, b, e)):
                assert torch.equal(g[first:first + e].cpu().double().transpose(0, 1), w)
            first += e


@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_borders_between_codes_and_ends_of_the_range(gpu, dtype):
    """Keys and values as they come (no rotation): on borders, beside them, at the ends of the exponents, at the type's ends."""
    cfg = config(q=2, kv=2, d=64, dtype=dtype, page=16, n_pages=20)
    step = Step(gpu, cfg, [0], [200], rope=False, in_f32=True)
    border = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0])
    x = border.repeat(200, 6 * 4)
    g = torch.Generator().manual_seed(1)
    x = x * torch.where(torch.rand(x.shape, generator=g) < 0.5, -1.0, 1.0)
    nudge = torch.randint(-1, 2, x.shape, generator=g)
    x = torch.where(nudge == 0, x, torch.nextafter(x, x + nudge))
    lo, hi = EXPONENTS[dtype]
    e = torch.randint(lo - 4, hi - 2, (200, 1), generator=g)
    e[:8, 0] = torch.tensor([lo - 20, lo - 3, lo - 2, lo - 1, lo, hi - 1, hi, 0])
    x = torch.ldexp(x, e)
    x[20:30] = torch.ldexp(torch.ones(()), torch.tensor(hi)) * 5.1       # saturates, or almost
    x[30] = 65519.0
    x[31] = 65520.0
    x[32] = 3.3895314e38
    x[33] = 3.3961776e38
    x[34] = torch.finfo(torch.float32).tiny
    x[35] = 1e-45
    step.qkv = x.contiguous()
    step.qkv_dev = step.qkv.to(gpu)
    step.write()
    rows = step.qkv.double().view(200, 6, 64).transpose(0, 1)
    k, v = held(cfg, step.dp.pool.cpu(), step.table, 0, 200)
    for got, want in ((k, rows[2:4]), (v, rows[4:])):
        want = quantised(want, dtype)[0]
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())


@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_rows_that_are_not_finite_are_stored_as_nan(gpu, dtype):
    cfg = config(dtype=dtype)
    step = Step(gpu, cfg, [0], [20], rope=False, in_f32=True)
    k0 = cfg.n_q_heads * cfg.head_dim
    v0 = k0 + cfg.n_kv_heads * cfg.head_dim
    step.qkv[2, k0 + 4] = math.nan
    step.qkv[5, v0 + 1] = math.inf
    step.qkv[7, v0 + 128] = -math.inf
    step.qkv[9, k0 + 100] = 1e6            # past fp16's range
    step.qkv_dev.copy_(step.qkv)
    step.write()
    want_k, want_v = torch.zeros(2, 20, dtype=torch.bool), torch.zeros(2, 20, dtype=torch.bool)
    want_k[0, 2] = want_v[0, 5] = want_v[1, 7] = True
    want_k[0, 9] = dtype == B.SPD_F16
    k_out, v_out = (torch.empty(20, 2, 128, device=gpu) for _ in range(2))
    B.spd_pages_read(step.dp.ctx, step.plan, step.dp.pool, k_out, v_out)
    k, v = held(cfg, step.dp.pool.cpu(), step.table, 0, 20)
    for x, want in ((k, want_k), (v, want_v), (k_out.cpu().transpose(0, 1), want_k), (v_out.cpu().transpose(0, 1), want_v)):
        assert torch.equal(torch.isnan(x).all(-1), want) and torch.equal(torch.isnan(x).any(-1), want)


@gpu_test
def test_rotated_keys_that_fp32_cannot_hold(gpu):
    """The rotation of two large features leaves 32 bits (and with them bf16): NaN, and nothing else is."""
    cfg = config(q=1, kv=1, d=64, page=16, n_pages=4)
    step = Step(gpu, cfg, [1], [3], in_f32=True)
    step.qkv[:] = 1.0
    step.qkv[1, 64:128] = 3.0e38            # a pair's length is 4.2e38
    step.qkv_dev.copy_(step.qkv)
    step.write()
    rope = step.rope.cpu().view(-1, 32, 2)
    want = quantised(rotate(step.qkv[:, 64:128].double().view(3, 1, 64), rope[1:4]), B.SPD_BF16)[0][:, 0]
    got = held(cfg, step.dp.pool.cpu(), step.table, 0, 4)[0][0, 1:]
    assert torch.isnan(want).any() and torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())


# ------------------------------------------------------------------------------------------ GPU: attention

@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("positions,q_lens", LENGTHS, ids=lambda v: "-".join(map(str, v)))
def test_write_then_attend(gpu, dtype, positions, q_lens):
    step = Step(gpu, config(dtype=dtype, page=32, n_pages=60), positions, q_lens, seed=len(positions) + sum(q_lens))
    step.write()
    check_attention(step, step.attend())


@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("q,kv,d,page", [(1, 1, 64, 16), (4, 4, 128, 16), (5, 5, 128, 64), (12, 4, 64, 128), (16, 1, 128, 256), (32, 2, 64, 32), (9, 3, 128, 64)])
def test_heads_and_pages(gpu, q, kv, d, page, dtype):
    cfg = config(q=q, kv=kv, d=d, page=page, n_pages=3 + 1200 // page, dtype=dtype)
    for positions, q_lens in (([77, 300], [40, 1]), ([300, 1], [2, 1])):
        step = Step(gpu, cfg, positions, q_lens, seed=q)
        step.write()
        check_attention(step, step.attend())


@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (16, 4), (33, 0), (64, 40), (100, 17), (1000, 4), (5, 600)])
@pytest.mark.parametrize("positions,q_lens", [([200, 3], [1, 1]), ([150], [90]), ([0, 400], [130, 20]), ([320], [3])], ids=str)
def test_window_and_sinks(gpu, dtype, window, sinks, positions, q_lens):
    step = Step(gpu, config(dtype=dtype, page=16, n_pages=60), positions, q_lens, window=window, sinks=sinks, seed=window)
    step.write()
    check_attention(step, step.attend())


@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("q_len", [1, 3, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_not_finite_reach_only_those_that_see_them(gpu, dtype, q_len, d):
    cfg = config(d=d, dtype=dtype, page=16, n_pages=60)
    width = (cfg.n_q_heads + 2 * cfg.n_kv_heads) * d
    key0, val0 = cfg.n_q_heads * d, (cfg.n_q_heads + cfg.n_kv_heads) * d

    def spoil(step, past):
        past[10, key0 + 3] = math.nan          # hidden from everyone: outside every window, no sink
        past[11, val0 + 5] = math.inf
        past[12, val0 + d + 7] = -math.inf     # head 1
        past[190, key0 + 7] = math.inf         # visible to the first of the chunk's queries only
        past[191, width - 1] = math.nan        # head 1
    step = Step(gpu, cfg, [200], [q_len], window=12, sinks=4, seed=3, spoil=spoil)
    step.write()
    got = step.attend()
    check_attention(step, got)
    assert torch.isnan(got[0]).any() and (q_len < 40 or not torch.isnan(got[12:]).any())


@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_len", [1, 30])
def test_pages_that_held_other_sequences(gpu, dtype, d, q_len):
    """Behind a sequence's end a page holds what was there: any codes, scales of rows that were not finite among them."""
    cfg = config(page=64, n_pages=4, dtype=dtype, d=d)
    step = Step(gpu, cfg, [70], [q_len], seed=5)
    g = torch.Generator().manual_seed(1)
    dirt = torch.randint(0, 256, step.dp.pool.shape, generator=g).to(torch.uint8)
    raw = dirt.view(cfg.n_pages, cfg.n_kv_heads, -1)
    raw[..., 64 * d:] = torch.where(torch.rand(raw[..., 64 * d:].shape, generator=g) < 0.5, 255, 110).to(torch.uint8)
    step.dp.pool.copy_(dirt.view(-1).to(gpu))
    past = torch.randn(70, step.qkv.shape[1], generator=torch.Generator().manual_seed(2)).to(T16[dtype]).to(gpu)
    B.spd_pages_write(step.dp.ctx, B.PagePlan(step.dp, [0], [70], step.table), past, step.rope, step.dp.pool)
    step.write()
    check_attention(step, step.attend())


@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
@pytest.mark.parametrize("q_len", [1, 33])
def test_scales_far_apart(gpu, dtype, q_len):
    """Groups and rows of very different magnitudes, down to the least scale: nothing underflows on the way that the type can hold."""
    cfg = config(dtype=dtype, page=16, n_pages=40)
    d, kv, nq = cfg.head_dim, cfg.n_kv_heads, cfg.n_q_heads

    def spoil(step, past):
        x = past.view(len(past), -1, d // 32, 32)
        g = torch.Generator().manual_seed(4)
        # keys stay of a size (scores with them); values' groups go from 2^-20 to 2^6
        x[:, nq + kv:] *= 2.0 ** torch.randint(-20, 7, (len(past), kv, d // 32, 1), generator=g)
        x[:, nq:nq + kv] *= 2.0 ** torch.randint(-6, 1, (len(past), kv, d // 32, 1), generator=g)
    step = Step(gpu, cfg, [333], [q_len], seed=8, spoil=spoil)
    step.write()
    check_attention(step, step.attend())


@gpu_test
def test_pool_beyond_32_bits(gpu):
    """Pages at the end of a pool of more than 4 GiB."""
    cfg = config(q=8, kv=8, d=128, page=256, n_pages=16000)
    n = cfg.n_pages
    order = [n - 1, 0, n - 2, 1, n - 3, 8000]
    step = Step(gpu, cfg, [300, 400], [1, 30], seed=2, order=order)
    assert step.dp.sizes.pool_bytes > 1 << 32
    step.write()
    got = step.attend()
    used = sorted(order)
    per = step.dp.pool.numel() // n
    small = torch.cat([step.dp.pool[i * per:(i + 1) * per] for i in used])
    step.cfg, step.table = config(q=8, kv=8, d=128, page=256, n_pages=len(used)), [[used.index(p) for p in row] for row in step.table]
    step.dp.pool = small
    check_attention(step, got)


@gpu_test
@pytest.mark.parametrize("dtype", TYPES, ids=TYPE_IDS)
def test_long_contexts_cut_into_parts(gpu, dtype):
    for positions, q_lens, over in (([20000], [1], {}), ([9000, 30, 4000], [1, 1, 1], {}), ([6000], [70], {}), ([5000], [40], dict(window=3000, sinks=20))):
        cfg = config(dtype=dtype, page=64, n_pages=340, max_ctx=20032, q=8, kv=2)
        step = Step(gpu, cfg, positions, q_lens, seed=q_lens[0], **over)
        step.write()
        check_attention(step, step.attend())


@gpu_test
def test_strided_rows_queries_in_place_and_a_graph(gpu):
    cfg = config(q=6, kv=3, d=64, page=16)
    step = Step(gpu, cfg, [20, 300], [37, 1], seed=9)
    plain = torch.empty_like(step.q)
    B.spd_pages_write(step.dp.ctx, step.plan, step.qkv_dev, step.rope, step.dp.pool, plain)
    wide = torch.zeros(38, step.qkv.shape[1] + 16, dtype=torch.bfloat16, device=gpu)
    big = torch.zeros(38, 512, dtype=torch.bfloat16, device=gpu)
    q, out = wide[:, :6 * 64], big[:, 64:64 + 6 * 64]

    def once():
        wide[:, :-16] = step.qkv_dev
        B.spd_pages_write(step.dp.ctx, step.plan, wide, step.rope, step.dp.pool, q)
        B.spd_pages_attention(step.dp.ctx, step.plan, q, step.dp.pool, out, step.plan.workspace)
    once()
    assert torch.equal(q, plain) and torch.equal(wide[:, 6 * 64:-16], step.qkv_dev[:, 6 * 64:])
    check_attention(step, out, q)
    assert not big[:, :64].any() and not big[:, 64 + 6 * 64:].any()
    want = big.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        once()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once()
    for _ in range(4):
        big.zero_()
        step.dp.pool.zero_()
        B.spd_pages_write(step.dp.ctx, B.PagePlan(step.dp, [0, 0], [20, 300], step.table), torch.randn(320, 768, device=gpu).to(torch.bfloat16), step.rope, step.dp.pool)
        graph.replay()
        torch.cuda.synchronize()
        again = big.clone()
        big.zero_()
        once()
        assert torch.equal(again, big) and not torch.equal(again, want)
