"""The 8-bit serving operators (include/spd_q8.h) at the edges of what a caller may hand them: tables, numbers and buffers that do not
fit, nothing to do, matrices that share memory, values at the ends of their types."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2502_20727_amd import binding as B

from test_q8_serving import KIND_IDS, KINDS, T16, U, U32, Step, check_rows, config, held, pages, reference, tables  # noqa: F401

gpu_test = pytest.mark.gpu


# ------------------------------------------------------------------------------------------ CPU: plans

@pytest.mark.parametrize("positions,q_lens,table", [([0], [1], [[]]), ([0, 0], [40, 1], [[1], [2, 3]]), ([64, 0], [1, 40], [[4, 5], [6, 7, 8]]),
                                                    ([0], [1], np.zeros((1, 0), np.int32))], ids=str)
def test_a_sequence_with_too_few_pages_is_refused(pages, positions, q_lens, table):
    """Another sequence's longer list lends it none: page 0 is not read or written for it."""
    _, ctx = pages()
    with pytest.raises(B.SpdError) as e:
        B.spd_pages_plan(ctx, positions, q_lens, table)
    assert e.value.code == B.SPD_EINVAL


@pytest.mark.parametrize("table", [[[1]], [[1], [2], [3]], []], ids=str)
def test_a_table_has_a_list_for_each_sequence(pages, table):
    _, ctx = pages()
    with pytest.raises(ValueError):
        B.spd_pages_plan(ctx, [0, 0], [1, 1], table)


FAR = 1 << 32


@pytest.mark.parametrize("over", [
    dict(positions=np.array([FAR])), dict(q_lens=np.array([FAR + 1])), dict(table=np.array([[FAR + 3]])), dict(table=[[np.int64(FAR + 3)]]),
    dict(table=[[FAR + 3]]), dict(positions=[FAR]), dict(window=FAR + 5), dict(window=8, sinks=FAR + 1), dict(window=FAR)], ids=str)
def test_numbers_beyond_32_bits_are_refused(pages, over):
    _, ctx = pages()
    a = dict(positions=[0], q_lens=[1], table=[[3]], window=0, sinks=0)
    a.update(over)
    with pytest.raises((ValueError, OverflowError)):
        B.spd_pages_plan(ctx, a["positions"], a["q_lens"], a["table"], a["window"], a["sinks"])


@pytest.mark.parametrize("over", [dict(positions=[0.5]), dict(q_lens=np.array([1.7])), dict(table=[[2.9]]), dict(table=np.array([[2.9]]))], ids=str)
def test_fractions_are_refused(pages, over):
    _, ctx = pages()
    a = dict(positions=[0], q_lens=[1], table=[[3]])
    a.update(over)
    with pytest.raises(TypeError):
        B.spd_pages_plan(ctx, a["positions"], a["q_lens"], a["table"])


def test_whole_numbers_of_any_type_make_the_same_plan(pages):
    _, ctx = pages()
    want = B.spd_pages_plan(ctx, [3, 40], [1, 2], [[7], [8, 9]])
    for t in (np.int64, np.uint8, np.int32):
        table = np.array([[7, 0], [8, 9]], t)
        assert np.array_equal(B.spd_pages_plan(ctx, np.array([3, 40], t), np.array([1, 2], t), table), want)
    assert np.array_equal(B.spd_pages_plan(ctx, torch.tensor([3, 40]), (1, 2), [(7,), np.array([8, 9])]), want)


# ------------------------------------------------------------------------------------------ CPU: packers

def test_scales_of_every_other_place_are_packed():
    K, N = 16, 700
    r = np.random.RandomState(0)
    codes, scale = r.randint(-127, 128, (K, N)).astype(np.int8), r.rand(2 * N).astype(np.float32)[::2]
    c, s = B.spd_q8_unpack(K, N, B.spd_q8_pack_codes(codes, scale))
    assert np.array_equal(s, scale) and np.array_equal(c, codes)


def test_packers_refuse_buffers_that_are_too_short():
    K, N = 70, 20
    need = B.spd_q8_weight_bytes(K, N)
    w, codes, scale = np.ones((K, N), np.float32), np.ones((K, N), np.int8), np.ones(N, np.float32)
    short, apart = np.zeros(need - 1, np.uint8), np.zeros(2 * need, np.uint8)[::2]
    for buf in (short, apart):
        for call in (lambda: B.spd_q8_pack(w, buf), lambda: B.spd_q8_pack_codes(codes, scale, buf), lambda: B.spd_q8_unpack(K, N, buf)):
            with pytest.raises(ValueError):
                call()
        assert not buf.any()
    whole = np.zeros(need, np.uint8)
    assert B.spd_q8_pack(w, whole) is whole and B.spd_q8_unpack(K, N, whole)[0].all()


# ------------------------------------------------------------------------------------------ nothing to do

def test_nothing_to_do_needs_no_addresses(pages):
    _, ctx = pages()
    lib, plan = B.lib(), B.spd_pages_plan(ctx, [], [], [])
    ph = plan.ctypes.data
    dev = (ph + 15) // 16 * 16                  # (never read)
    assert lib.spd_pages_write(ctx, ph, dev, B.SPD_BF16, None, 1536, None, None, None, 0, None) == B.SPD_OK
    assert lib.spd_pages_read(ctx, ph, dev, None, B.SPD_F32, None, None, None) == B.SPD_OK
    assert lib.spd_pages_attention(ctx, ph, dev, None, 1024, None, None, 1024, None, None) == B.SPD_OK
    for rows, n in ((0, 8), (2, 0)):
        assert lib.spd_q8_norm(B.SPD_F32, rows, n, None, 8, None, 0, None, 1e-5, None, 0, None, 8, None, None) == B.SPD_OK
        assert lib.spd_q8_rows(B.SPD_F32, rows, n, None, 8, None, 8, None, None) == B.SPD_OK
        assert lib.spd_q8_swiglu(B.SPD_F32, rows, n, None, 16, None, 8, None, None) == B.SPD_OK
    assert lib.spd_q8_matmul(0, 32, 8, None, 32, None, None, B.SPD_F32, None, 0, None, 8, None, None) == B.SPD_OK
    # what is wrong without any work is still wrong
    assert lib.spd_pages_write(ctx, ph, dev, B.SPD_F16, None, 1536, None, None, None, 0, None) == B.SPD_EINVAL
    assert lib.spd_q8_rows(5, 0, 8, None, 8, None, 8, None, None) == B.SPD_EINVAL
    assert lib.spd_q8_matmul(0, 0, 8, None, 32, None, None, B.SPD_F32, None, 0, None, 8, None, None) == B.SPD_EINVAL


@gpu_test
def test_empty_tensors(gpu):
    cfg = config()
    dp = B.DevicePages(cfg, gpu)

    def none(n, t=torch.bfloat16, rows=0):
        return torch.empty(rows, n, dtype=t, device=gpu)
    plan = B.PagePlan(dp, [3, 0], [0, 0], [[1], []])
    B.spd_pages_write(dp.ctx, plan, none(1536), dp.rope, dp.pool, none(1024))
    B.spd_pages_attention(dp.ctx, plan, none(1024), dp.pool, none(1024), plan.workspace)
    plan = B.PagePlan(dp, [], [], [])
    k, v = (torch.empty(0, 2, 128, device=gpu) for _ in range(2))
    B.spd_pages_read(dp.ctx, plan, dp.pool, k, v)
    for rows, n in ((0, 16), (3, 0)):
        codes, scales = none(n, torch.int8, rows), torch.full((rows,), 7.0, device=gpu)
        B.spd_q8_norm(none(n, rows=rows), None, torch.ones(n, device=gpu), 1e-5, None, codes, scales)
        B.spd_q8_rows(none(n, rows=rows), codes, scales)
        B.spd_q8_swiglu(none(2 * n, rows=rows), codes, scales)
        assert bool((scales == 7.0).all())
    packed = torch.from_numpy(B.spd_q8_pack(np.ones((16, 16), np.float32))).to(gpu)
    B.spd_q8_matmul(none(16, torch.int8), torch.empty(0, device=gpu), packed, 16, None, none(16))


# ------------------------------------------------------------------------------------------ matrices that share memory

def test_rotated_queries_share_no_memory_with_what_others_read(pages):
    """Keys and values of other workgroups, queries but not in their place, rows of another stride."""
    _, ctx = pages()
    lib, a = B.lib(), np.zeros(1 << 16, np.uint8)
    base = (a.ctypes.data + 255) // 256 * 256
    plan = B.spd_pages_plan(ctx, [0], [2], [[0]])
    ph, w = plan.ctypes.data, (8 + 4) * 128
    for ld, qo, ldq in ((w, base + 2 * 1024, w), (w, base + 2 * 128, w), (w, base + 2 * 1024, 1024), (2 * w, base + 2 * (w - 128), 2 * w),
                        (2 * w, base + 2 * (2 * w - 512), 2 * w)):
        assert lib.spd_pages_write(ctx, ph, base, B.SPD_BF16, base, ld, base, base, qo, ldq, None) == B.SPD_EINVAL, (ld, qo - base, ldq)
    assert lib.spd_pages_write(ctx, ph, base, B.SPD_F32, base, w, base, base, base + 4 * w, 1024, None) == B.SPD_EINVAL


@gpu_test
def test_rotated_queries_beside_what_they_are_made_of(gpu):
    """In rows of one buffer, behind the values, they share no memory with them."""
    step = Step(gpu, config(q=4, kv=2, page=16), [20], [37], seed=9)
    step.write()
    wide = torch.zeros(37, 1024 + 512, dtype=torch.bfloat16, device=gpu)
    wide[:, :1024] = step.qkv_dev
    B.spd_pages_write(step.dp.ctx, step.plan, wide[:, :1024], step.rope, step.dp.pool, wide[:, 1024:])
    assert torch.equal(wide[:, 1024:], step.q) and torch.equal(wide[:, :1024], step.qkv_dev)


@gpu_test
@pytest.mark.parametrize("q_len", [1, 3, 40])
def test_attention_into_the_columns_of_the_keys(gpu, q_len):
    """Rows of queries, keys and values whose keys and values are put away already take the output in their place: it shares no memory with
    the queries beside it."""
    step = Step(gpu, config(q=4, kv=4, page=16, n_pages=80), [600, 0], [q_len, 2], seed=q_len)
    step.write()
    want = step.attend()
    wide = torch.zeros(q_len + 2, 3 * 512, dtype=torch.bfloat16, device=gpu)
    wide[:, :512] = step.q
    B.spd_pages_attention(step.dp.ctx, step.plan, wide[:, :512], step.dp.pool, wide[:, 512:1024], step.plan.workspace)
    assert torch.equal(wide[:, :512], step.q) and torch.equal(wide[:, 512:1024], want) and not wide[:, 1024:].any()
    with pytest.raises(B.SpdError):
        B.spd_pages_attention(step.dp.ctx, step.plan, wide[:, :512], step.dp.pool, wide[:, 256:768], step.plan.workspace)


def test_rows_and_products_reject_matrices_that_share_memory():
    """Sums and outputs in the place of a summand are fine, on a part of one they are not, nor are codes on what they are made of."""
    lib, a = B.lib(), np.zeros(1 << 16, np.uint8)
    base = (a.ctypes.data + 255) // 256 * 256
    far = base + 8192
    norm = dict(x=base, ldx=64, add=far, lda=64, s=far + 8192, lds=64, c=far + 16384, ldc=64)
    for over in (dict(s=base + 4), dict(s=base + 256), dict(s=far + 128), dict(s=base, lds=64, x=base + 4, ldx=64), dict(c=base), dict(c=far + 64),
                 dict(c=far + 8192 + 4), dict(s=base + 256 - 64, lds=128)):
        x = {**norm, **over}
        assert lib.spd_q8_norm(B.SPD_F32, 3, 64, x["x"], x["ldx"], x["add"], x["lda"], far + 24576, 1e-5, x["s"], x["lds"], x["c"], x["ldc"],
                               far + 28672, None) == B.SPD_EINVAL, over
    assert lib.spd_q8_rows(B.SPD_F32, 3, 64, base, 64, base + 64, 64, far, None) == B.SPD_EINVAL
    assert lib.spd_q8_swiglu(B.SPD_F32, 3, 32, base, 64, base + 64, 64, far, None) == B.SPD_EINVAL
    for add, lda, out, ldo, codes in ((base, 64, base + 16, 64, far), (base, 64, base + 256, 64, far), (None, 0, far, 64, far), (None, 0, far + 64, 64, far)):
        assert lib.spd_q8_matmul(3, 64, 64, codes, 64, far + 8192, far + 16384, B.SPD_F32, add, lda, out, ldo, None, None) == B.SPD_EINVAL, (out - base)


@gpu_test
def test_rows_and_products_side_by_side_in_one_buffer(gpu):
    """Columns of one buffer are as good as buffers of their own; sums and outputs in place of a summand too."""
    g = torch.Generator().manual_seed(0)
    wide = torch.randn(5, 96, generator=g).to(gpu)
    x, add, total = wide[:, :32], wide[:, 32:64], wide[:, 64:]
    gain = torch.ones(32, device=gpu)
    codes, scales = torch.empty(5, 32, dtype=torch.int8, device=gpu), torch.empty(5, device=gpu)
    want = x + add
    B.spd_q8_norm(x, add, gain, 1e-5, total, codes, scales)
    assert torch.equal(total, want)
    again, scales2 = torch.empty_like(codes), torch.empty_like(scales)
    for into in (x, add):
        kept = wide.clone()
        B.spd_q8_norm(x, add, gain, 1e-5, into, again, scales2)
        assert torch.equal(into, want) and torch.equal(again, codes) and torch.equal(scales2, scales)
        wide.copy_(kept)
    packed = torch.from_numpy(B.spd_q8_pack(np.eye(32, dtype=np.float32))).to(gpu)
    out = torch.empty(5, 32, device=gpu)
    B.spd_q8_matmul(codes, scales, packed, 32, add, out)
    B.spd_q8_matmul(codes, scales, packed, 32, add, total)
    assert torch.equal(total, out)
    B.spd_q8_matmul(codes, scales, packed, 32, add, add)
    assert torch.equal(add, out)


# ------------------------------------------------------------------------------------------ GPU: ends of the types

@gpu_test
@pytest.mark.parametrize("dtype,cache", KINDS, ids=KIND_IDS)
@pytest.mark.parametrize("blank,position,q_len", [(4608, 5000, 1), (4608, 5000, 3), (800, 1000, 60), (3200, 3300, 1)])
def test_positions_of_scale_zero(gpu, dtype, cache, blank, position, q_len):
    """Pages as the cleared pool holds them (codes and scales 0) are keys and values of zeros like any others."""
    cfg = config(q=4, kv=2, page=16, n_pages=330, max_ctx=5200, dtype=dtype, cache=cache)
    step = Step(gpu, cfg, [0], [0], seed=1)
    width, g = 8 * 128, torch.Generator().manual_seed(blank + q_len)
    step.table = tables(cfg, [position + q_len], 1)
    past = torch.randn(position - blank, width, generator=g).to(T16[dtype]).to(gpu)
    B.spd_pages_write(step.dp.ctx, B.PagePlan(step.dp, [blank], [position - blank], step.table), past, step.rope, step.dp.pool)
    step.positions, step.q_lens, step.ends = [position], [q_len], [position + q_len]
    step.plan = B.PagePlan(step.dp, [position], [q_len], step.table)
    step.qkv_dev = torch.randn(q_len, width, generator=g).to(T16[dtype]).to(gpu)
    step.q = torch.empty(q_len, 4 * 128, dtype=T16[dtype], device=gpu)
    step.write()
    want, mag = reference(step, step.q.cpu(), step.dp.pool.cpu())
    got = step.attend().cpu().double()
    t = T16[dtype]
    bound = (U[t] * 1.01 + 2e-5) * mag + U[t] * want.abs() * 1.01 + 2.0 ** -24
    if dtype == B.SPD_F16:         # a weight below fp16's normal numbers is off by 2^-25 of the largest weight
        k, v = held(cfg, step.dp.pool.cpu(), step.table, 0, position + q_len)
        s = torch.einsum("nhd,hpd->hnp", step.q.cpu().double().view(q_len, 4, 128), k.repeat_interleave(2, 0)) / math.sqrt(128)
        hidden = torch.arange(position + q_len) > torch.arange(position, position + q_len)[:, None]
        w = s.masked_fill(hidden, -math.inf).softmax(-1).amax(-1)                                         # [4, q_len]
        bound = bound + ((position + q_len) * 2.0 ** -25 * w.t() * float(v.abs().max())).repeat_interleave(128, 1)
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).nan_to_num(9e9).max())


@gpu_test
@pytest.mark.parametrize("n", [64, 5000, 8192, 20000])
@pytest.mark.parametrize("add", [False, True])
def test_norm_of_rows_whose_squares_leave_32_bits(gpu, n, add):
    """The sum of squares is beyond fp32, or below it, the values and the norm are not."""
    g = torch.Generator().manual_seed(n)
    x = torch.randn(6, n, generator=g) * torch.tensor([1e18, 1e20, 3e30, 1e37, 1e-22, 1e-30])[:, None]
    y = x.flip(1) * 0.5 if add else None
    gain = 1 + 0.1 * torch.randn(n, generator=g)
    codes, scales = torch.empty(6, n, dtype=torch.int8, device=gpu), torch.empty(6, device=gpu)
    for eps in (0.0, 1e-5):
        B.spd_q8_norm(x.to(gpu), None if y is None else y.to(gpu), gain.to(gpu), eps, None, codes, scales)
        s = x.double() if y is None else x.double() + y.double()
        v = s / (s.square().mean(-1, keepdim=True) + eps).sqrt() * gain.double()
        # as for rows of ordinary size: a sum of n squares, at most n / 256 of them one after the other, ten levels of partial sums
        check_rows(codes, scales, v, (n / 256 + 26) * U32)


# ------------------------------------------------------------------------------------------ CPU: how chunks are cut

@pytest.mark.parametrize("over,batch,n,at,window,sinks,parts", [
    (dict(q=5, kv=5), 3, 333, 5001, 0, 0, 99), (dict(q=5, kv=5), 3, 333, 5001, 2048, 4, 45), (dict(q=64, kv=8), 1, 300, 2000, 0, 0, 57),
    (dict(q=40, kv=40), 1, 73, 1850, 0, 0, 6), (dict(q=12, kv=4, d=64), 1, 1056, 1365, 0, 0, 120), (dict(q=10, kv=10), 6, 574, 7661, 0, 0, 36),
    (dict(q=40, kv=40), 1, 151, 0, 0, 0, 0)], ids=str)
def test_chunks_are_cut_as_was_fastest(pages, over, batch, n, at, window, sinks, parts):
    """The cut that took least of three that were timed on the device (partial results of all pieces)."""
    cfg, ctx = pages(page=64, n_pages=batch * 140, max_ctx=9000, **over)
    table = [list(range(140 * b, 140 * b + 140)) for b in range(batch)]
    size = B.spd_pages_plan_get_info(ctx, B.spd_pages_plan(ctx, [at] * batch, [n] * batch, table, window, sinks)).workspace_bytes
    assert max(0, size - 16384 * 4) // (128 * cfg.n_kv_heads * (cfg.head_dim + 2) * 4) == parts
