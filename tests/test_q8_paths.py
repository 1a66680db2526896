"""Every kernel of the 8-bit product, with the ways it has of storing its results, and the attention of every pair of types, where the types' own code
parts: against plain computations in 64 bits."""
import math

import pytest
import torch

from paper_2502_20727_amd import binding as B

from test_q8_serving import KIND_IDS, KINDS, T16, TYPES, U, U32, Step, config, held, reference

gpu_test = pytest.mark.gpu

FAR = (1 << 22) + 16        # bytes between rows of codes that are too many for offsets inside a panel

# kernel of spd_q8_kernel_of(): rows, K, N.  One, two, three and many k-tiles (a stage is one or two), whole and short last ones, widths that end
# inside a tile and a group of four columns.
PATHS = [
    (1, (1, 1, 64)), (1, (16, 192, 1280)), (1, (15, 640, 516)), (2, (257, 64, 257)), (2, (16, 640, 7168)), (3, (41, 640, 5120)), (3, (41, 65, 4100)), (4, (500, 130, 257)),
    (4, (480, 1024, 264)), (5, (257, 448, 1000)), (5, (260, 1728, 1024)),
    (6, (700, 64, 64)), (6, (333, 1728, 5120)), (6, (700, 130, 1000)), (6, (1000, 192, 516)), (7, (6932, 65, 257)), (7, (6932, 320, 264)), (7, (6800, 130, 260)),
    (8, (6932, 1, 516)), (8, (6932, 130, 520)), (8, (1087, 1728, 5120)), (8, (6932, 192, 513)),
    (9, (4096, 1, 2056)), (9, (4090, 128, 2056)), (9, (4096, 130, 2052)), (9, (2855, 1376, 4096)), (9, (4000, 256, 2057)),
    (10, (4096, 64, 4100)), (10, (6932, 544, 2794)), (10, (4090, 192, 4104)), (10, (4500, 320, 4096)),
    (11, (2100, 7168, 4096)), (11, (2050, 7232, 4100)), (12, (4090, 7201, 4104)), (12, (4500, 7168, 4096))]
FAR_PATHS = [(1, 64, 16), (5, 100, 50), (3, 1, 1), (33, 130, 260), (70, 704, 72)]


@pytest.mark.parametrize("kernel,shape", PATHS, ids=str)
def test_shapes_reach_their_kernels(kernel, shape):
    assert B.spd_q8_kernel_of(*shape) == kernel


def test_every_kernel_is_reached():
    assert {k for k, _ in PATHS} == set(range(1, 13))
    assert all(B.spd_q8_kernel_of(*s, FAR) == 0 for s in FAR_PATHS)


@pytest.mark.parametrize("rows,K,N,ld", [(0, 64, 16, 64), (-1, 64, 16, 64), (1, 0, 16, 64), (1, B.SPD_Q8_MAX_K + 1, 16, 1 << 20), (1, 64, 0, 64), (1, 64, 16, 48)])
def test_kernel_of_rejects(rows, K, N, ld):
    with pytest.raises(B.SpdError) as e:
        B.spd_q8_kernel_of(rows, K, N, ld)
    assert e.value.code == B.SPD_EINVAL


def inputs(dev, rows, K, N, ld, seed):
    """Codes of any value, scales that leave products of about unit size; the exact products."""
    g = torch.Generator(device=dev).manual_seed(seed)
    a = torch.zeros(rows, ld, dtype=torch.int8, device=dev)
    a[:, :min(ld, (K + 15) // 16 * 16)] = torch.randint(-127, 128, (rows, min(ld, (K + 15) // 16 * 16)), generator=g, device=dev).to(torch.int8)
    w = torch.randint(-127, 128, (K, N), generator=g, device=dev).to(torch.int8)
    sa = 0.1 + torch.rand(rows, generator=g, device=dev)
    sw = (0.1 + torch.rand(N, generator=g, device=dev)) / (5000 * math.sqrt(K))
    packed = torch.from_numpy(B.spd_q8_pack_codes(w.cpu().numpy(), sw.cpu().numpy())).to(dev)
    exact = (a[:, :K].double() @ w.double()) * sa.double()[:, None] * sw.double()      # (whole numbers far below 2^53)
    return a[:, :K], sa, packed, exact, g


def check(out, p, y, t, what):
    """The sum in fp32, two scales, a summand, the rounding to the type.  fp16's least step is 2^-24."""
    want = p if y is None else p + y.double()
    bound = 4 * U32 * p.abs() + 2 * U32 * want.abs() + U[t] * want.abs() * 1.0001 + 2.0 ** -25
    err = (out.double() - want).abs()
    assert bool((err <= bound).all()), (what, float((err / bound).max()))


def stores(a, sa, packed, p, g, t, what):
    """Outputs by themselves, in rows with a gap, in rows that keep no alignment; without a summand, with one, in its place."""
    rows, N = p.shape
    y = torch.randn(rows, N, generator=g, device=p.device).to(t)
    for gap in (0, 4, 8, 3):
        for add in (False, True):
            wide = torch.full((rows, N + gap), 5.0, dtype=t, device=p.device)
            out = wide[:, :N]
            B.spd_q8_matmul(a, sa, packed, N, y if add else None, out)
            check(out, p, y if add else None, t, (what, gap, add))
            assert bool((wide[:, N:] == 5.0).all()), (what, gap, add)
        place = torch.full((rows, N + gap), 5.0, dtype=t, device=p.device)
        place[:, :N] = y
        B.spd_q8_matmul(a, sa, packed, N, place[:, :N], place[:, :N])
        assert torch.equal(place, torch.cat([out, wide[:, N:]], 1)), (what, gap, "in place")


@gpu_test
@pytest.mark.parametrize("kernel,shape", PATHS, ids=str)
def test_product_of_every_kernel(gpu, kernel, shape):
    rows, K, N = shape
    a, sa, packed, p, g = inputs(gpu, rows, K, N, (K + 15) // 16 * 16, rows + K)
    for t in TYPES.values():
        stores(a, sa, packed, p, g, t, (kernel, shape, t))


@gpu_test
@pytest.mark.parametrize("shape", FAR_PATHS, ids=str)
def test_product_of_rows_far_apart(gpu, shape):
    rows, K, N = shape
    a, sa, packed, p, g = inputs(gpu, rows, K, N, FAR, rows + K)
    for t in TYPES.values():
        stores(a, sa, packed, p, g, t, (shape, t))


@gpu_test
@pytest.mark.parametrize("rows,K,N", [(5, 300, 40), (200, 640, 520), (2100, 192, 1027)])
def test_products_beyond_fp16_are_infinities_of_their_sign(gpu, rows, K, N):
    a, sa, packed, p, _ = inputs(gpu, rows, K, N, (K + 15) // 16 * 16, 1)
    sa, p = sa * 1e5, p * 0
    out32, out = torch.empty(rows, N, device=gpu), torch.empty(rows, N, dtype=torch.float16, device=gpu)
    B.spd_q8_matmul(a, sa, packed, N, None, out32)
    B.spd_q8_matmul(a, sa, packed, N, None, out)
    beyond, within = out32.abs() > 65536, out32.abs() < 65504
    assert beyond.any() and within.any()
    assert torch.equal(out[beyond].float(), out32[beyond].sign() * math.inf)
    assert bool(((out.float() - out32).abs()[within] <= U[torch.float16] * out32.abs()[within] * 1.0001 + 2.0 ** -25).all())


# ------------------------------------------------------------------------------------------ attention

def check_closely(step, got, q=None, more=0.0):
    """As close as the pool's type allows: a weight is rounded to it once, and below fp16's normal numbers by 2^-25 of the largest weight.  Beside e4m3 fp16's
    weights are probabilities times the values' scales, so that the largest is that of a probability times a row's largest value.  more: what the scores' own rounding moves a probability by."""
    q = (step.q if q is None else q).cpu()
    cfg, pool, t = step.cfg, step.dp.pool.cpu(), T16[step.cfg.dtype]
    want, mag = reference(step, q, pool)
    got = got.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    d, group, first, floor = cfg.head_dim, cfg.n_q_heads // cfg.n_kv_heads, 0, torch.zeros_like(want)
    if t is torch.float16:
        for b, (p, n) in enumerate(zip(step.positions, step.q_lens)):
            k, v = held(cfg, pool, step.table, b, p + n)
            x = q[first:first + n].double().view(n, cfg.n_q_heads, d)
            at, key = torch.arange(p, p + n)[:, None], torch.arange(p + n)[None]
            hidden = key > at
            if step.window:
                hidden |= (key <= at - step.window) & (key >= step.sinks)
            for h in range(cfg.n_q_heads):
                size = v[h // group].abs().amax(-1).nan_to_num(0.0)
                w = (x[:, h] @ k[h // group].t() / math.sqrt(d)).masked_fill(hidden, -math.inf).softmax(-1).nan_to_num(0.0)
                most = (w * size).amax(-1) if cfg.cache_dtype == B.SPD_E4M3 else w.amax(-1) * size.max()
                floor[first:first + n, h * d:(h + 1) * d] = ((p + n) * 2.0 ** -25 * most)[:, None]
            first += n
    ok = ~torch.isnan(want)
    bound = (U[t] * 1.01 + 2e-5 + more) * mag + U[t] * want.abs() * 1.01 + 2.0 ** -24 + floor
    err = (got - want).abs()
    assert bool((err[ok] <= bound[ok]).all()), float((err / bound)[ok].max())


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 3), (33, 0), (64, 40), (100, 17), (1000, 4), (5, 600)])
@pytest.mark.parametrize("positions,q_lens", [([200, 3], [1, 1]), ([150], [90]), ([0, 400], [130, 20]), ([320], [3]), ([900, 600], [1, 3])], ids=str)
def test_window_and_sinks_of_every_kind(gpu, dtype, cache, window, sinks, positions, q_lens):
    step = Step(gpu, config(dtype=dtype, cache=cache, page=16, n_pages=110), positions, q_lens, window=window, sinks=sinks, seed=window)
    step.write()
    check_closely(step, step.attend())


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("q_len", [1, 3, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_not_finite_in_every_kind(gpu, dtype, cache, q_len, d):
    cfg = config(d=d, dtype=dtype, cache=cache, page=16, n_pages=60)
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
    check_closely(step, got)
    assert torch.isnan(got[0]).any() and (q_len < 40 or not torch.isnan(got[12:]).any())


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("q_len", [1, 30])
def test_pages_that_held_other_sequences_in_every_kind(gpu, dtype, cache, q_len):
    """Behind a sequence's end a page holds what was there: finite codes, NaN scales."""
    cfg = config(page=64, n_pages=4, dtype=dtype, cache=cache)
    step = Step(gpu, cfg, [70], [q_len], seed=5)
    w = 1 if cache == B.SPD_E4M3 else 2
    dirt = torch.randint(0, 120, step.dp.pool.shape, generator=torch.Generator().manual_seed(1)).to(torch.uint8)      # (finite in all three types)
    raw = dirt.view(cfg.n_pages, cfg.n_kv_heads, -1)
    raw[..., 2 * 64 * 128 * w:] = 255                       # every scale NaN
    step.dp.pool.copy_(dirt.view(-1).to(gpu))
    past = torch.randn(70, step.qkv.shape[1], generator=torch.Generator().manual_seed(2)).to(T16[dtype]).to(gpu)
    B.spd_pages_write(step.dp.ctx, B.PagePlan(step.dp, [0], [70], step.table), past, step.rope, step.dp.pool)
    step.write()
    check_closely(step, step.attend())


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("q,kv,d,page", [(1, 1, 64, 16), (5, 5, 128, 64), (12, 4, 64, 128), (16, 1, 128, 256), (9, 3, 128, 32)])
def test_heads_and_lengths_of_every_kind(gpu, dtype, cache, q, kv, d, page):
    cfg = config(q=q, kv=kv, d=d, page=page, n_pages=6 + 1900 // page, dtype=dtype, cache=cache)
    step = Step(gpu, cfg, [77, 300, 0, 980], [40, 1, 16, 2], seed=q)
    step.write()
    check_closely(step, step.attend())


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_maxima_that_move_along_the_keys(gpu, dtype, cache, up, d):
    """Scores that rise, with room in a tile and without, or fall, beside values whose sizes go the other way."""
    cfg = config(q=4, kv=2, d=d, page=16, n_pages=60, dtype=dtype, cache=cache)

    def spoil(step, past):
        f = torch.linspace(0.1, 5.0, past.shape[0])[:, None].to(past.dtype)
        past[:, 4 * d:6 * d] *= f if up else f.flip(0)
        past[:, 6 * d:] *= f.flip(0) if up else f
    step = Step(gpu, cfg, [400, 390], [90, 1], seed=3, spoil=spoil)
    step.write()
    # a score of up to s (in units of e) is a sum of d products in fp32, at most 16 of them one after the other, and three factors: 20 u s off, and
    # a probability, with the sum that it is divided by, by twice as much
    k = torch.cat([held(cfg, step.dp.pool.cpu(), step.table, b, step.ends[b])[0].flatten(0, 1) for b in range(2)])
    s = float(step.q.float().cpu().view(-1, d).norm(dim=-1).max() * k.norm(dim=-1).max()) / math.sqrt(d)
    check_closely(step, step.attend(), more=2 * 20 * U32 * s)


@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("batch,kv,d,prefix,lone", [(40, 8, 64, 9008, 0), (33, 8, 128, 8336, 0), (2100, 8, 64, 32, 3000), (300, 2, 128, 800, 4000)])
def test_more_sequences_than_workgroups(gpu, dtype, cache, batch, kv, d, prefix, lone):
    """Sequences that are not cut into parts, so that a wave goes through more blocks than it keeps pages of at a time; more of them, times heads, than there are
    counters for parts, one much longer than the rest.  All but that one share their first pages."""
    held_of = -(-(max(prefix, lone) + 16) // 16)
    cfg = config(q=2 * kv, kv=kv, d=d, page=16, n_pages=2 * held_of + batch, dtype=dtype, cache=cache, max_ctx=9100)
    dp = B.DevicePages(cfg, gpu)
    g, t = torch.Generator().manual_seed(batch), T16[dtype]
    common, own = list(range(prefix // 16)), list(range(held_of, 2 * held_of))
    table = [common + [2 * held_of + b] for b in range(batch)]
    positions = [prefix] * batch
    if lone:
        table[batch // 2], positions[batch // 2] = own, lone
    width = 4 * kv * d
    past = torch.randn(prefix + lone, width, generator=g).to(t).to(gpu)
    B.spd_pages_write(dp.ctx, B.PagePlan(dp, [0, 0], [prefix, lone], [common, own]), past, dp.rope, dp.pool)
    plan = B.PagePlan(dp, positions, [1] * batch, table)
    qkv = torch.randn(batch, width, generator=g).to(t).to(gpu)
    q, out = torch.empty(batch, 2 * kv * d, dtype=t, device=gpu), torch.full((batch, 2 * kv * d), math.nan, dtype=t, device=gpu)
    B.spd_pages_write(dp.ctx, plan, qkv, dp.rope, dp.pool, q)
    B.spd_pages_attention(dp.ctx, plan, q, dp.pool, out, plan.workspace)
    assert not torch.isnan(out).any()
    some = sorted({0, batch // 2, batch - 1, batch // 3})

    class Part:
        pass
    part = Part()
    part.cfg, part.dp, part.window, part.sinks = cfg, dp, 0, 0
    part.positions, part.q_lens, part.table = [positions[b] for b in some], [1] * len(some), [table[b] for b in some]
    check_closely(part, out[some], q[some])
