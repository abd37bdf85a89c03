"""Attention over pages with any workspace up to what it says it needs: long and short sequences, forks, the same results within the
tolerances, and nothing written behind the workspace."""

from __future__ import annotations

import pytest
import torch

from gpu_pages import BF16, Pool, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("forks", [False, True], ids=["apart", "forks"])
@pytest.mark.parametrize("H,G", [(1, 4), (8, 2), (2, 20)])
def test_any_workspace(H, G, forks, fp8):
    p = Pool(seqs=9, pages=500, most=130, P=16, L=1, H=H, fp8=fp8)
    p.extend([0, 1, 2, 3, 4], [1900, 3, 0, 700, 1201])
    seqs = [4, 0, 1, 2, 3, 0]
    if forks:
        p.fork([0, 0, 0, 4], [5, 6, 7, 8], [800, 1500, 640, 1000])
        p.extend([5, 6, 7, 8], [3, 40, 1, 17])
        seqs = [5, 0, 1, 8, 6, 2, 4, 7, 3]
    q = torch.randn(len(seqs), H * G, 128, generator=p.g).to(BF16).cuda()
    need = p.pages.attention_workspace(q, seqs)
    assert need > 0
    room = torch.empty(need + 4096, dtype=torch.uint8, device="cuda")
    for part in (need, need - 16, need * 15 // 16, need * 3 // 4, need // 2, need // 3, need // 8, need // 40, 16):
        part = part // 16 * 16
        room.fill_(255)  # (of a state that is read and not written: NaN)
        out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
        p.pages.attention(0, q, out, seqs, lse=lse, workspace=room[:part])
        check_attention(p, 0, q, out, lse, seqs, what=f"workspace {part} of {need}")
        assert bool((room[part:] == 255).all()), part
