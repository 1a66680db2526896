"""Every kernel of the 8-bit product, with the ways it has of storing its results, against plain computations in 64 bits."""
import math

import pytest
import torch

from paper_2502_20727_amd import binding as B

from test_q8_serving import TYPES, U, U32

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
