"""Refusals of the rotary positions and of the pages: every check runs on the host before any GPU work (the pointers below are
never used)."""

import ctypes

import numpy as np
import pytest

from paper_2607_15621_amd import fsx

PTR = 1 << 20  # an address that no check dereferences
INVALID, UNSUPPORTED = 1, 2


def rotate(x=PTR, y=PTR + (1 << 24), pos=PTR, rows=10, axis=None, freq=None, null=False, **kw):
    plan = fsx.RotaryPlan([0] * 64 if axis is None else axis, [1.0] * 64 if freq is None else freq)
    d = dict(dtype=fsx.BF16, n_heads=4, head_dim=128, n_pairs=64, layout=0, n_axes=1, inverse=0, axis=plan.c_axis, freq=plan.c_freq,
             x_row=512, x_head=128, y_row=512, y_head=128, pos_axis=10, pos_row=1)
    d.update(kw)
    desc = fsx.RotaryDesc(*(d[n] for n, _ in fsx.RotaryDesc._fields_))
    return fsx.lib().fsx_rotary_rows(None if null else ctypes.byref(desc), x, y, pos, rows, None), fsx.last_error()


@pytest.mark.parametrize("kw,code,word", [
    (dict(null=True), INVALID, "desc"), (dict(dtype=fsx.FP8_E4M3), UNSUPPORTED, "BF16"), (dict(n_heads=0), INVALID, "n_heads"),
    (dict(n_heads=4097), INVALID, "n_heads"), (dict(head_dim=1), INVALID, "head_dim"), (dict(head_dim=1025), INVALID, "head_dim"),
    (dict(n_pairs=0), INVALID, "n_pairs"), (dict(n_pairs=129, head_dim=512), INVALID, "n_pairs"), (dict(head_dim=126), INVALID, "n_pairs"),
    (dict(layout=2), INVALID, "layout"), (dict(n_axes=0), INVALID, "n_axes"), (dict(n_axes=257), INVALID, "n_axes"),
    (dict(inverse=2), INVALID, "inverse"), (dict(axis=[0] * 63 + [1]), INVALID, "axis of pair 63"),
    (dict(axis=[-1] + [0] * 63), INVALID, "axis of pair 0"), (dict(freq=[1.0] * 63 + [float("nan")]), INVALID, "freq of pair 63"),
    (dict(freq=[float("inf")] + [1.0] * 63), INVALID, "freq of pair 0"), (dict(freq=[2.0 ** 20 + 1] + [1.0] * 63), INVALID, "freq"),
    (dict(x_row=-1), INVALID, "strides"), (dict(pos_axis=(1 << 30) + 1), INVALID, "strides"), (dict(rows=-1), INVALID, "n_rows"),
    (dict(rows=(1 << 26) + 1), UNSUPPORTED, "2^26"), (dict(x=0), INVALID, "non-NULL"), (dict(y=0), INVALID, "non-NULL"),
    (dict(pos=0), INVALID, "non-NULL"), (dict(x=PTR + 1), INVALID, "aligned"), (dict(dtype=fsx.F32, y=PTR + (1 << 24) + 2), INVALID, "aligned"),
    (dict(pos=PTR + 2), INVALID, "aligned"), (dict(y_head=64), INVALID, "overlap"), (dict(y_row=500), INVALID, "overlap"),
    (dict(y_row=0), INVALID, "overlap"), (dict(y=PTR, y_row=1024), INVALID, "same strides"), (dict(y=PTR, x_head=136), INVALID, "same strides"),
    (dict(y=PTR + 256), INVALID, "x and y overlap"), (dict(y=PTR + 1024), INVALID, "x and y overlap"),
    (dict(y=PTR - 256), INVALID, "x and y overlap"),
    (dict(x_row=1024, y_row=1024, y=PTR + 2 * 511), INVALID, "x and y overlap"),   # begins before the row's heads end
    (dict(x_row=1024, y_row=1024, y=PTR + 2 * 513), INVALID, "x and y overlap"),   # and runs into the next row
    (dict(x_row=1024, y_row=2048, y=PTR + 2 * 512), INVALID, "x and y overlap")])
def test_rotary(kw, code, word):
    got, msg = rotate(**kw)
    assert got == code and word in msg, msg


def test_rotary_without_rows_needs_no_gpu():
    assert rotate(rows=0, x=0, y=0, pos=0)[0] == 0


def test_rotary_plans():
    plan = fsx.RotaryPlan.sections((2, 3), base=16.0)
    assert plan.axis.tolist() == [0, 0, 1, 1, 1] and np.allclose(plan.freq, 16.0 ** -(np.arange(5) / 5))
    plan = fsx.RotaryPlan.sections((2, 0, 4), base=16.0, joint=False)
    assert plan.axis.tolist() == [0, 0, 2, 2, 2, 2] and np.allclose(plan.freq, [1, 0.25, 1, 0.5, 0.25, 0.125])
    with pytest.raises(ValueError):
        fsx.RotaryPlan([0], [1.0, 2.0])


def create(**kw):
    d = dict(dtype=fsx.FP8_E4M3, n_layers=2, n_kv_heads=4, head_dim=128, page_rows=16, n_pages=10, max_seqs=4, max_seq_pages=8, k=PTR, v=PTR,
             k_scale=PTR, v_scale=PTR)
    d.update(kw)
    cfg, out = fsx.PagesCfg(*(d[n] for n, _ in fsx.PagesCfg._fields_)), ctypes.c_void_p(5)
    code = fsx.lib().fsx_pages_create(ctypes.byref(cfg), None, ctypes.byref(out))
    assert not out.value
    return code, fsx.last_error()


@pytest.mark.parametrize("kw,code,word", [
    (dict(dtype=fsx.F32), UNSUPPORTED, "BF16"), (dict(n_layers=0), INVALID, "n_layers"), (dict(n_layers=1025), INVALID, "n_layers"),
    (dict(n_kv_heads=0), INVALID, "n_kv_heads"), (dict(n_kv_heads=1025), INVALID, "n_kv_heads"), (dict(head_dim=96), UNSUPPORTED, "head_dim"),
    (dict(n_layers=1024, n_kv_heads=65), UNSUPPORTED, "2^16"), (dict(page_rows=8), INVALID, "page_rows"), (dict(page_rows=48), INVALID, "page_rows"), (dict(page_rows=512), INVALID, "page_rows"),
    (dict(n_pages=0), INVALID, "n_pages"), (dict(n_pages=2 ** 31 - 1, n_layers=1024, n_kv_heads=64, page_rows=256), INVALID, "2^48"),
    (dict(max_seqs=0), INVALID, "max_seqs"), (dict(max_seqs=65537), INVALID, "max_seqs"),
    (dict(max_seq_pages=0), INVALID, "max_seq_pages"), (dict(max_seq_pages=(1 << 24) + 1), INVALID, "max_seq_pages"),
    (dict(max_seq_pages=1 << 24, max_seqs=17), INVALID, "max_seq_pages"), (dict(k=0), INVALID, "k and v"), (dict(v=PTR + 8), INVALID, "k and v"),
    (dict(k_scale=0), INVALID, "scale"), (dict(v_scale=PTR + 4), INVALID, "scale")])
def test_create(kw, code, word):
    got, msg = create(**kw)
    assert got == code and word in msg, msg


def test_nulls():
    L, one = fsx.lib(), (ctypes.c_int32 * 1)(0)
    big, need, out = (ctypes.c_int64 * 1)(0), ctypes.c_int64(5), ctypes.c_void_p(5)
    assert L.fsx_pages_create(None, None, ctypes.byref(out)) == INVALID and not out.value
    assert L.fsx_pages_create(None, None, None) == INVALID
    assert L.fsx_pages_extend(None, 1, one, one, None) == INVALID and "pages" in fsx.last_error()
    assert L.fsx_pages_fork(None, 1, one, one, None, None) == INVALID
    assert L.fsx_pages_keep(None, 1, one, one, one, one, None) == INVALID
    assert L.fsx_pages_free(None, 1, one, None) == INVALID
    assert L.fsx_pages_tables(None, None, None, None) == INVALID
    assert L.fsx_pages_write(None, None, PTR, PTR, 1, one, big, big, None) == INVALID
    assert L.fsx_pages_attention(None, None, 0, PTR, PTR, None, 1, one, None, 0, None) == INVALID
    assert L.fsx_pages_attention_workspace(None, None, 1, one, ctypes.byref(need)) == INVALID and need.value == 0
    assert L.fsx_pages_attention_workspace(None, None, 1, one, None) == INVALID
    L.fsx_pages_destroy(None)


@pytest.mark.parametrize("values", [
    [1 << 32], (-(1 << 31) - 1,), [np.int64((1 << 32) + 1)], [np.array((1 << 32) + 1)], [np.array([1 << 31])], np.array([1 << 32]), [3e9],
    range(1 << 33, (1 << 33) + 2),
])
def test_numbers_outside_32_bits(values):
    for a in ([(values[0], 1)], [(0, values[0])]):
        with pytest.raises(ValueError, match="outside 32 bits"):
            fsx.RowRanges([a])


@pytest.mark.parametrize("values", [[0, (1 << 31) - 1], (np.int64(5), 7), np.array([3, 4], np.int64), [np.array(9), 2], range(2)])
def test_numbers_of_32_bits(values):
    r = fsx.RowRanges([[(x, x) for x in values]])
    assert r.first.dtype == np.int32 and r.first.tolist() == r.count.tolist() == [int(x) for x in values] and r.counts.tolist() == [len(values)]
