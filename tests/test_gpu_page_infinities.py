"""Attention over pages: an infinite value reaches its channel as long as its weight is not zero in fp32."""

from __future__ import annotations

import math

import numpy as np
import pytest
import torch

from gpu_pages import BF16, Pool

pytestmark = pytest.mark.gpu

SCALE = float(np.float32(math.log(2)))  # scores in log2 units are q.k itself


@pytest.mark.parametrize("G", [1, 4, 20])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("whole", [True, False], ids=["powers", "others"])
def test_an_infinite_value_of_a_tiny_weight(whole, D, G):
    """Sequence i has 48 rows of score 0 but for one, whose score in log2 units is -i, or -i - 1/2; its value is infinite in one
    channel.  A weight of 2^-125 or more is a number of fp32: infinity times it is infinite, and no other channel sees it.  (A power
    of two is a bf16 value: its second half is zero but for what keeps it above.)"""
    assert np.float32(SCALE) * np.float32(1.4426950408889634) == np.float32(1.0)
    n = 126 if whole else 125
    p = Pool(seqs=n, pages=3 * n, most=3, P=16, L=1, H=1, D=D)
    p.extend(list(range(n)), [48] * n)
    p.k.zero_()
    table, _ = p.pages.tables()
    q = torch.zeros(n, G, D)
    q[..., 0] = 1.0
    k, v = p.k.cpu(), p.v.cpu()
    for i in range(n):
        row = (7 * i) % 48
        page = table[i, row // 16]
        score = -i if whole else -i - 0.5
        k[0, page, 0, row % 16, 0], k[0, page, 0, row % 16, 1] = round(score), score - round(score)
        v[0, page, 0, row % 16, (5 * i) % D] = math.inf if i % 2 else -math.inf
    p.k.copy_(k)
    p.v.copy_(v)
    q[..., 1] = 1.0
    out = torch.empty(n, G, D, dtype=BF16, device="cuda")
    p.pages.attention(0, q.to(BF16).cuda(), out, list(range(n)), scale=SCALE)
    out = out.float().cpu()
    wrong = []
    for i in range(n):
        c, want = (5 * i) % D, math.inf if i % 2 else -math.inf
        if not bool((out[i, :, c] == want).all()) or not bool(torch.isfinite(torch.cat([out[i, :, :c], out[i, :, c + 1:]], 1)).all()):
            wrong.append(i)
    assert not wrong, wrong
