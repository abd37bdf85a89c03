"""Attention over pages refuses tensors that some of its workgroups would write while others have still to read them, and takes heads
that lie between each other's."""

from __future__ import annotations

import pytest
import torch

from gpu_pages import BF16, F32, Pool, check_attention
from paper_2607_15621_amd import fsx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_refused(fp8):
    p = Pool(seqs=3, pages=80, most=70, L=1, fp8=fp8)
    p.extend([0, 1], [700, 33])
    arena = torch.zeros(1 << 16, dtype=F32, device="cuda")
    half = arena.view(BF16)
    q = half[:2 * 4 * 128].view(2, 4, 128)
    q.copy_(torch.randn(2, 4, 128, generator=p.g))
    out, lse, ws = torch.empty_like(q), torch.empty(2, 4, device="cuda"), torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    room = arena.view(torch.uint8)
    assert 0 < p.pages.attention_workspace(q, [0, 1]) <= 1 << 16
    before = [t.clone() for t in (arena, p.k.view(torch.uint8), p.v.view(torch.uint8), *([p.ks.view(torch.uint8), p.vs.view(torch.uint8)] if fp8 else []))]
    into_pool = p.k.view(torch.uint8).reshape(-1)
    cases = [
        ("out must not overlap q", dict(out=q)),
        ("out must not overlap q", dict(out=half[8:8 + 1024].view(2, 4, 128))),               # begins within a head
        ("out must not overlap q", dict(out=half[512:512 + 1024].view(2, 4, 128))),           # begins with the last row
        ("out must not overlap q", dict(out=half[512 + 384:].as_strided((2, 4, 128), (2048, 128, 1), 896))),
        ("out must not overlap q", dict(out=arena[:1024].view(2, 4, 128))),                   # of another type
        ("out must not lie in the pool", dict(out=into_pool[:2048].view(BF16).view(2, 4, 128))),
        ("out must not lie in the pool", dict(out=p.v.view(torch.uint8).reshape(-1)[-2048:].view(BF16).view(2, 4, 128))),
        ("lse must not overlap q", dict(lse=arena[511:519].view(2, 4))),
        ("lse must not overlap out", dict(lse=out.view(F32).reshape(-1)[504:512].view(2, 4))),
        ("lse must not lie in the pool", dict(lse=into_pool[:32].view(F32).view(2, 4))),
        ("workspace must not overlap q", dict(workspace=room[16:1 << 16])),
        ("workspace must not overlap out", dict(out=half[1 << 15:(1 << 15) + 1024].view(2, 4, 128), workspace=room[1 << 12:(1 << 12) + (1 << 16)])),
        ("workspace must not overlap lse", dict(lse=arena[2048:2056].view(2, 4), workspace=room[1 << 12:(1 << 12) + (1 << 15)])),
        ("workspace must not lie in the pool", dict(workspace=into_pool[:1 << 15])),
    ]
    if fp8:
        cases += [("out must not lie in the pool", dict(out=p.ks.view(BF16).reshape(-1)[:1024].view(2, 4, 128))),
                  ("lse must not lie in the pool", dict(lse=p.vs.reshape(-1)[-8:].view(2, 4))),
                  ("workspace must not lie in the pool", dict(workspace=p.vs.view(torch.uint8).reshape(-1)[:4096]))]
    for word, kw in cases:
        a = dict(out=out, lse=lse, workspace=ws)
        a.update(kw)
        with pytest.raises(fsx.FsxError, match=word) as e:
            p.pages.attention(0, q, a["out"], [0, 1], lse=a["lse"], workspace=a["workspace"])
        assert e.value.code == 1
    torch.cuda.synchronize()
    for t, b in zip((arena, p.k.view(torch.uint8), p.v.view(torch.uint8), *([p.ks.view(torch.uint8), p.vs.view(torch.uint8)] if fp8 else [])), before):
        assert torch.equal(t.view(torch.uint8), b.view(torch.uint8))
    p.pages.attention(0, q, out, [0, 1], lse=lse, workspace=ws)
    check_attention(p, 0, q, out, lse, [0, 1])


def test_side_by_side_in_one_buffer():
    """Queries, outputs, log sums and workspace of one buffer: heads of the outputs behind the queries' in a row, between them, and
    rows of the one between rows of the other."""
    p = Pool(seqs=5, pages=120, most=90, L=1)
    p.extend([0, 1, 2, 3, 4], [1300, 33, 0, 1, 260])
    seqs = [4, 0, 2, 1, 3]
    n, H, D = 5, 4, 128
    values = torch.randn(n, H, D, generator=p.g).to(BF16)
    for what in ("behind", "between", "rows", "packed"):
        room = torch.full((1 << 20,), 3.0, dtype=BF16, device="cuda")
        if what == "behind":
            both = room[:n * 2 * H * D].view(n, 2, H, D)
            q, out, used = both[:, 0], both[:, 1], n * 2 * H * D
        elif what == "between":
            both = room[:n * 2 * H * D].view(n, H, 2, D)
            q, out, used = both[:, :, 0], both[:, :, 1], n * 2 * H * D
        elif what == "rows":  # (a longer row of the one)
            q = room.as_strided((n, H, D), (4 * H * D, D, 1), 0)
            out = room.as_strided((n, H, D), (8 * H * D, D, 1), H * D)
            used = 8 * n * H * D
        else:
            q, out, used = room[:n * H * D].view(n, H, D), room[n * H * D:2 * n * H * D].view(n, H, D), 2 * n * H * D
        q.copy_(values)
        need = p.pages.attention_workspace(q, seqs)
        lse = room[used:used + 2 * n * H].view(F32).view(n, H)
        at = (used + 2 * n * H + 7) // 8 * 8
        ws = room[at:at + need // 2].view(torch.uint8)
        p.pages.attention(0, q, out, seqs, lse=lse, workspace=ws)
        assert torch.equal(q.cpu(), values), what
        assert bool((room[at + need // 2:] == 3.0).all()), what
        check_attention(p, 0, values, out, lse, seqs, what=what)
