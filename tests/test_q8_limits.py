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
