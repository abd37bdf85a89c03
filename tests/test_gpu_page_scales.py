"""Rows to be written into fp8 pages that lie in the pool's scales, which the call writes too, are refused."""

from __future__ import annotations

import pytest
import torch

from gpu_pages import BF16, Pool
from paper_2607_15621_amd import fsx

pytestmark = pytest.mark.gpu


def test_rows_in_the_scales():
    p = Pool(seqs=3, pages=64, most=10, L=1, H=2, P=16, fp8=True)
    p.extend([0], [20])
    p.pages.extend([1], [3])
    before = [t.clone() for t in (p.k, p.v, p.ks, p.vs)]
    k, v = (t.cuda() for t in p.new(3))
    for scales in (p.ks, p.vs):
        flat = scales.view(-1)
        for within in (flat[:768].view(1, 3, 2, 128), flat.view(BF16)[-768:].view(1, 3, 2, 128)):
            pairs = [(within, within)]
            if within.dtype is BF16:
                pairs += [(within, v), (k, within)]
            for a, b in pairs:
                with pytest.raises(fsx.FsxError, match="must not lie in the pool") as e:
                    p.pages.write(0, 1, a, b, [1], fsx.PackedRows([3]))
                assert e.value.code == 1
    torch.cuda.synchronize()
    for t, b in zip((p.k, p.v, p.ks, p.vs), before):
        assert torch.equal(t.view(torch.uint8), b.view(torch.uint8))
    p.pages.write(0, 1, k, v, [1], fsx.PackedRows([3]))
    p.rows[1] = p.stored(k.cpu(), v.cpu())
    p.check()
