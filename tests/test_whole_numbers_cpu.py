"""Lists of sequences, rows, lengths and axes: whole numbers in whatever form, and fractions refused instead of cut off."""

import numpy as np
import pytest
import torch

from paper_2607_15621_amd import fsx

FRACTIONS = [[2.7], [0.9, 1.2], np.array([0.5]), np.array([1.0, 2.5], np.float32), [1, 2.000001], (-0.5,), [float("nan")], [float("inf")],
             np.array([np.nan]), [-np.inf], torch.tensor([1.5]), [torch.tensor(0.25)], ["3"], [None], [1 + 2j], [1 + 0j], np.array(["7"])]
WHOLE = [[2, 3], (2, 3), np.array([2, 3]), np.array([2.0, 3.0]), [2.0, 3.0], [np.int64(2), 3], [np.array(2), 3.0], range(2, 4),
         torch.tensor([2, 3]), [torch.tensor(2), torch.tensor(3)], np.array([2, 3], np.uint64), np.array([2, 3], np.int8), np.array([2, 9, 3])[::2],
         np.array([2, 3], object), np.array([[2], [3]])]


@pytest.mark.parametrize("values", FRACTIONS, ids=repr)
def test_fractions(values):
    for call in (lambda: fsx._int32s(values, "seqs"), lambda: fsx.PackedRows(values), lambda: fsx.PackedRows([0] * len(values), values),
                 lambda: fsx.RotaryPlan(values, [1.0] * len(values)), lambda: fsx.RotaryPlan.sections(values)):
        with pytest.raises(ValueError, match="whole numbers"):
            call()
    x = values[0] if len(values) == 1 else values[1]
    for a in ([(x, 1)], [(0, x)]):
        with pytest.raises(ValueError, match="whole numbers"):
            fsx.RowRanges([a])


@pytest.mark.parametrize("values", WHOLE, ids=repr)
def test_whole_numbers(values):
    a, address = fsx._int32s(values, "seqs")
    assert a.dtype == np.int32 and a.tolist() == [2, 3] and address == a.ctypes.data and a.flags.c_contiguous
    rows = fsx.PackedRows(values)
    assert rows.len.dtype == np.int64 and rows.len.tolist() == [2, 3] and rows.start.tolist() == [0, 2]
    assert fsx.PackedRows([1, 1], values).start.tolist() == [2, 3]
    plan = fsx.RotaryPlan(values, [1.0, 2.0])
    assert plan.axis.dtype == np.int32 and plan.axis.tolist() == [2, 3]
    assert fsx.RotaryPlan.sections(values).axis.tolist() == [0, 0, 1, 1, 1]


def test_no_numbers():
    for empty in ([], (), np.array([]), np.array([], np.int32), range(0)):
        a, _ = fsx._int32s(empty, "seqs")
        assert a.dtype == np.int32 and a.size == 0 and fsx.PackedRows(empty).n == 0


def test_what_a_program_keeps_is_not_shared():
    """Later changes of the array do not reach a plan or the rows that were made from it."""
    a = np.array([2, 3], np.int64)
    rows, plan = fsx.PackedRows(a, a), fsx.RotaryPlan(a.astype(np.int32), [1.0, 2.0])
    a[:] = 7
    assert rows.len.tolist() == rows.start.tolist() == plan.axis.tolist() == [2, 3]


@pytest.mark.parametrize("values", [[1 << 63], [-(1 << 63) - 1], [2.0 ** 63], np.array([1 << 63], np.uint64), [1 << 70], [1e300]])
def test_numbers_outside_64_bits(values):
    for call in (lambda: fsx.PackedRows(values), lambda: fsx.PackedRows([0], values)):
        with pytest.raises(ValueError, match="outside 64 bits"):
            call()
    for call in (lambda: fsx._int32s(values, "seqs"), lambda: fsx.RotaryPlan(values, [1.0])):
        with pytest.raises(ValueError, match="outside 32 bits"):
            call()


def test_axes_outside_32_bits():
    for values in ([1 << 32], np.array([1 << 32]), [-(1 << 31) - 1]):
        with pytest.raises(ValueError, match="outside 32 bits"):
            fsx.RotaryPlan(values, [1.0])
