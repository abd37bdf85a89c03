"""A pool whose keys, values and scales overlap is refused, on the host before any GPU work (the pointers below are never used):
keys and values are moved by workgroups of their own, and one would read what the other has moved already."""

import ctypes

import pytest
import torch

from paper_2607_15621_amd import fsx

INVALID = 1
AT, CODES, SCALES = 1 << 24, 2 * 10 * 4 * 16 * 128, 2 * 10 * 4 * 16 * 4


def create(**kw):
    d = dict(dtype=fsx.FP8_E4M3, n_layers=2, n_kv_heads=4, head_dim=128, page_rows=16, n_pages=10, max_seqs=4, max_seq_pages=8, k=AT, v=AT + CODES,
             k_scale=AT + 2 * CODES, v_scale=AT + 2 * CODES + SCALES)
    d.update(kw)
    cfg, out = fsx.PagesCfg(*(d[n] for n, _ in fsx.PagesCfg._fields_)), ctypes.c_void_p(5)
    code = fsx.lib().fsx_pages_create(ctypes.byref(cfg), None, ctypes.byref(out))
    assert not out.value
    return code, fsx.last_error()


@pytest.mark.parametrize("kw", [
    dict(v=AT), dict(v=AT + CODES - 16), dict(v=AT - CODES + 16), dict(k_scale=AT), dict(k_scale=AT + CODES - 16), dict(v_scale=AT + 2 * CODES - 16),
    dict(v_scale=AT + 2 * CODES), dict(v_scale=AT + 2 * CODES + SCALES - 16), dict(k_scale=AT - SCALES + 16),
    dict(dtype=fsx.BF16, k_scale=0, v_scale=0), dict(dtype=fsx.BF16, k_scale=0, v_scale=0, v=AT)], ids=repr)
def test_overlap(kw):
    code, msg = create(**kw)
    assert code == INVALID and "must not overlap" in msg, msg


@pytest.mark.skipif(torch.cuda.is_available(), reason="would make a handle")
@pytest.mark.parametrize("kw", [dict(), dict(v=AT - CODES), dict(dtype=fsx.BF16, v=AT + 2 * CODES, k_scale=0, v_scale=0),
                                dict(dtype=fsx.BF16, v=AT + 2 * CODES, k_scale=AT, v_scale=AT)], ids=repr)
def test_no_overlap(kw):
    """Past the checks: what is refused here is the missing device.  (Pages of bf16 have no scales.)"""
    code, msg = create(**kw)
    assert code not in (0, INVALID), msg
