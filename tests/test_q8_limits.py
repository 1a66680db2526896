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
