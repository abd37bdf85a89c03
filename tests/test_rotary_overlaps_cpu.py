"""Positions that lie in the rotary positions' output are refused: a workgroup would write what another has still to read.  On the
host, before any GPU work (the pointers below are never used)."""

import ctypes

import pytest
import torch

from paper_2607_15621_amd import fsx

Y = 1 << 24  # 10 rows of 4 heads of 128 bf16 channels, in rows of 1,024 elements
INVALID = 1


def rotate(pos, pos_axis=10, pos_row=1, axis=(0,) * 64, x=1 << 20, **kw):
    plan = fsx.RotaryPlan(axis, [1.0] * 64)
    d = dict(dtype=fsx.BF16, n_heads=4, head_dim=128, n_pairs=64, layout=0, n_axes=3, inverse=0, axis=plan.c_axis, freq=plan.c_freq,
             x_row=1024, x_head=128, y_row=1024, y_head=128, pos_axis=pos_axis, pos_row=pos_row)
    d.update(kw)
    desc = fsx.RotaryDesc(*(d[n] for n, _ in fsx.RotaryDesc._fields_))
    return fsx.lib().fsx_rotary_rows(ctypes.byref(desc), x, Y, pos, 10, None), fsx.last_error()


SECTIONS = (0,) * 20 + (1,) * 20 + (2,) * 24


@pytest.mark.parametrize("kw", [
    dict(pos=Y), dict(pos=Y, x=Y), dict(pos=Y - 4), dict(pos=Y - 36), dict(pos=Y + 9 * 2048 + 1020), dict(pos=Y + 1020, pos_row=512),
    dict(pos=Y + 1024, pos_row=511),                             # runs into the next row
    dict(pos=Y - 40, axis=SECTIONS), dict(pos=Y - 80, axis=SECTIONS), dict(pos=Y + 1024, pos_axis=256, axis=SECTIONS, pos_row=0),
    dict(pos=Y + 1000, y_head=256, n_heads=3), dict(pos=Y - 4 * ((1 << 30) - 1), pos_axis=(1 << 30) - 1, axis=(1,) * 64)], ids=repr)
def test_overlap(kw):
    code, msg = rotate(**kw)
    assert code == INVALID and "positions and y overlap" in msg, msg


@pytest.mark.skipif(torch.cuda.is_available(), reason="would launch")
@pytest.mark.parametrize("kw", [
    dict(pos=Y - 40), dict(pos=Y + 9 * 2048 + 1024), dict(pos=Y + 1024), dict(pos=Y + 1024, pos_row=512), dict(pos=Y - 40, axis=(0,) * 63 + (2,), pos_axis=5000),
    dict(pos=Y - 80, axis=(0,) * 32 + (1,) * 32),               # (axis 2 has no pair)
    dict(pos=Y + 512, y_head=512, n_heads=2, pos_row=512),       # behind a head
    dict(pos=Y + 1024, pos_axis=120, pos_row=512, axis=SECTIONS)], ids=repr)
def test_no_overlap(kw):
    """Past the checks: what is refused here is the missing device."""
    code, msg = rotate(**kw)
    assert code not in (0, INVALID), msg
