"""Pages: sequences extended, forked, pruned and freed, and rows written into them, bit for bit against sequences kept on the host."""

from __future__ import annotations

import math
import random

import numpy as np
import pytest
import torch

from gpu_pages import BF16, F32, FP8, U8, Pool, encode
from paper_2607_15621_amd import fsx

pytestmark = pytest.mark.gpu
kinds = pytest.mark.parametrize("fp8,D", [(False, 128), (False, 64), (True, 128), (True, 64)], ids=["bf16-128", "bf16-64", "fp8-128", "fp8-64"])


@kinds
@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["from-bf16", "from-f32"])
def test_rows_written(fp8, D, P, dtype):
    p = Pool(seqs=6, pages=60, most=20, P=P, D=D, fp8=fp8, H=3)
    p.extend([4, 1], [P + 3, 1], dtype)
    p.check()
    p.extend([0, 4, 5, 1], [2 * P, P - 4, 0, 1], dtype)  # up to a page's end, nothing, one more row
    p.extend([4, 0], [1, 1], dtype)
    p.check()


@kinds
def test_layers_strides_and_order(fp8, D):
    """A layer at a time out of a projection's rows, sequences out of order in the packed rows, gaps between them."""
    p = Pool(L=3, H=4, D=D, fp8=fp8, P=32)
    p.extend([0, 1, 2], [5, 40, 31], write=False)
    k, v = p.new(100)
    lens, starts = [31, 5, 39], [60, 3, 10]
    wide = torch.randn(3, 100, 6 + 8, D).to(BF16).cuda()
    wide[:, :, 6:10], wide[:, :, 10:] = k.cuda(), v.cuda()
    before = wide.clone()
    rows = fsx.PackedRows(lens, starts)
    for layer in (2, 0, 1):
        p.pages.write(layer, 1, wide[layer:layer + 1, :, 6:10], wide[layer:layer + 1, :, 10:], [2, 0, 1], rows)
    assert torch.equal(wide, before)
    table, length = p.pages.tables()
    got, (row_k, row_v) = (p.k.cpu(), p.v.cpu()), (encode(k)[0], encode(v)[0]) if fp8 else (k, v)
    for s, n, a in zip([2, 0, 1], lens, starts):
        for r in range(n):
            i = int(length[s]) - n + r
            for t, want in zip(got, (row_k, row_v)):
                assert torch.equal(t[:, table[s, i // 32], :, i % 32], want[:, a + r]), (s, r)
    first = got[0][:, table[1, 0], :, 0]  # sequence 1's first row was not written
    assert bool((first == 0x7F).all()) if fp8 else bool(first.isnan().all())
    # heads before rows
    hk, hv = (t.transpose(1, 2).contiguous().transpose(1, 2).cuda() for t in (k, v))
    p.pages.write(1, 2, hk[1:], hv[1:], [1], fsx.PackedRows([40], [0]))
    table, _ = p.pages.tables()
    for r in (0, 31, 32, 39):
        want = encode(k)[0] if fp8 else k
        assert torch.equal(p.k.cpu()[1:, table[1, r // 32], :, r % 32], want[1:, r])


def test_fp8_rows_of_every_kind():
    """Zeros, infinities, NaN of both signs, tiny and huge rows, bf16 and fp32."""
    for dtype in (F32, BF16):
        p = Pool(L=1, H=1, fp8=True, P=16, pages=4, most=2)
        x = torch.randn(1, 20, 1, 128, generator=p.g)
        x[0, 1] = 0.0
        x[0, 2] = -0.0
        x[0, 3, 0, 7], x[0, 3, 0, 100] = math.inf, -math.inf
        x[0, 4, 0, 0], x[0, 4, 0, 127] = math.nan, -math.nan
        x[0, 5] = math.nan
        x[0, 6] = math.inf
        x[0, 7] *= 1e-38
        x[0, 8] *= 1e-42
        x[0, 9] *= 1e38 / 4
        x[0, 10] = torch.linspace(-448, 448, 128)
        x[0, 11] = 3.0
        x[0, 12, 0, 5] = 1e30
        x = x.to(dtype)
        p.pages.extend([0], [20])
        p.pages.write(0, 1, x.cuda(), (-x).cuda(), [0], fsx.PackedRows([20]))
        for t, sc, src in ((p.k, p.ks, x), (p.v, p.vs, -x)):
            code, scale = encode(src)
            assert torch.equal(t[0, :2, 0].reshape(32, 128)[:20].cpu(), code[0, :, 0])
            assert torch.equal(sc[0, :2, 0].reshape(32)[:20].cpu(), scale[0, :, 0])


@kinds
@pytest.mark.parametrize("P", [16, 128])
def test_forks_diverge(fp8, D, P):
    p = Pool(seqs=12, pages=80, most=6, P=P, D=D, fp8=fp8, L=3)
    p.extend([0], [P + 7])
    p.fork([0] * 5, [1, 2, 3, 4, 5])
    p.check()
    p.extend([1, 3, 0, 2], [1, P, 2 * P, 3])
    p.check()
    p.fork([1, 3], [6, 7], [P + 3, 0])  # a shorter history; none
    p.extend([6, 7, 5], [1, 1, 1])
    p.check()
    p.free([0, 1])
    p.extend([4], [1])  # the shared page's last sharer keeps it
    p.check()
    p.free([2, 3, 4, 5, 6, 7, 8])
    assert p.pages.free_pages() == 80
    p.extend([0], [2 * P])
    p.check()


@kinds
@pytest.mark.parametrize("ranges", [[(0, 50)], [(0, 16), (32, 60)], [(1, 91)], [(3, 5), (20, 1), (21, 4), (40, 52)], [(0, 0)], [(91, 1)], [],
                                    [(i, 1) for i in range(0, 92, 2)], [(0, 17), (18, 74)]], ids=lambda r: str(r[:4]))
def test_rows_kept(fp8, D, ranges):
    p = Pool(seqs=6, pages=60, most=20, P=16, D=D, fp8=fp8)
    p.extend([0, 1, 2], [92, 100, 92])
    p.fork([1], [3])
    p.keep([0, 3], [ranges, ranges])  # in place; off shared pages
    p.check()
    p.keep([1], [ranges])  # pages that the fork left
    p.check()
    p.extend([0, 1, 3], [20, 20, 20])
    p.check()


@kinds
def test_long_rows_kept(fp8, D):
    """Many stretches of a workgroup, 256 ranges, several sequences in a call."""
    p = Pool(seqs=3, pages=200, most=100, P=32, D=D, fp8=fp8, L=1, H=1)
    p.extend([0, 1, 2], [2500, 1300, 900])
    r = random.Random(5)
    some = []
    for n in (2500, 1300):
        cut = sorted(r.sample(range(n), 512))
        some.append([(a, b - a) for a, b in zip(cut[::2], cut[1::2])])
    p.keep([0, 2, 1], [some[0], [(0, 3), (5, 895)], some[1]])
    p.check()


@pytest.mark.parametrize("seed", range(6))
def test_random_calls(seed):
    r = random.Random(seed)
    P = r.choice([16, 32])
    p = Pool(pages=50, seqs=6, most=8, L=r.choice([1, 2]), H=r.choice([1, 3]), P=P, D=r.choice([64, 128]), fp8=r.random() < 0.5)
    for _ in range(25):
        some = r.sample(range(6), r.randint(1, 4))
        try:
            what = r.choice(["extend", "extend", "fork", "keep", "keep", "free"])
            if what == "extend":
                p.extend(some, [min(r.choice([1, 3, P, 2 * P + 1]), 8 * P - len(p.rows[s])) for s in some])
            elif what == "fork":
                dst = [s for s in some if not p.rows[s]]
                src = [s for s in range(6) if s not in dst]
                if src:
                    p.fork([r.choice(src) for _ in dst], dst)
            elif what == "keep":
                ranges = []
                for s in some:
                    cut = sorted(r.randint(0, len(p.rows[s])) for _ in range(r.choice([2, 4, 8])))
                    ranges.append([(a, b - a) for a, b in zip(cut[::2], cut[1::2])])
                p.keep(some, ranges)
            else:
                p.free(some[:2])
        except fsx.FsxError as e:
            assert e.code == 3  # too few pages: nothing changed
        p.check()


def test_other_rows_stay():
    """Rows of the pool that no call should touch keep their bits."""
    p = Pool(seqs=4, pages=20, most=8, P=16)
    p.k.normal_()
    p.v.normal_()
    before = p.k.clone(), p.v.clone()
    p.extend([0, 1], [20, 16])
    p.fork([0], [2])
    p.extend([2], [1])
    p.keep([0], [[(2, 18)]])
    written = torch.zeros(20, 16, dtype=torch.bool)
    table, _ = p.pages.tables()
    written[table[1, 0]] = True
    written[[0, 1, 2, 3]] = True                # sequences 0 and 1, before
    written[1, 4:] = written[table[2, 1], 5:] = False
    assert table[0].tolist()[:2] == [4, 1] and table[2].tolist()[:2] == [0, 3]
    written[4] = True                           # page 0 was shared: sequence 0's rows moved to another
    for t, b in zip((p.k, p.v), before):
        same = (t == b).all(4).all(2).all(0).cpu()
        assert bool(same[~written].all()), (~same & ~written).nonzero()


def test_the_device_s_length_counts_in_a_replay():
    """A captured write goes to the rows that extend made room for since."""
    p = Pool(seqs=3, pages=20, most=8, L=1)
    p.extend([0, 1], [15, 3])
    p.pages.extend([0, 1], [1, 1])
    k, v = (t.cuda() for t in p.new(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        p.pages.write(0, 1, k, v, [0, 1], fsx.PackedRows([1, 1]))
        with pytest.raises(fsx.FsxError, match="captured") as e:
            p.pages.extend([0], [1])
        assert e.value.code == 2
        for call in (lambda: p.pages.free([0]), lambda: p.pages.fork([0], [2]), lambda: p.pages.keep([0], [[(0, 1)]])):
            with pytest.raises(fsx.FsxError, match="captured"):
                call()
    for step in range(4):
        if step:
            p.pages.extend([0, 1], [1, 1])
            nk, nv = p.new(2)
            k.copy_(nk)
            v.copy_(nv)
        graph.replay()
        torch.cuda.synchronize()
        for s, row in zip((0, 1), p.stored(k.cpu(), v.cpu())):
            p.rows[s].append(row)
        p.check()


def test_handles_made_and_given_back_while_a_graph_is_captured():
    p, gone = Pool(seqs=3, pages=20, most=8, L=1), Pool(seqs=3, pages=20, most=8, L=1)
    p.extend([0], [5])
    k, v = (t.cuda() for t in p.new(1))
    p.pages.extend([0], [1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        p.pages.write(0, 1, k, v, [0], fsx.PackedRows([1]))
        with pytest.raises(fsx.FsxError, match="captured"):
            fsx.Pages(p.k, p.v, 3, 8)
        gone.pages.close()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    p.rows[0] += p.stored(k.cpu(), v.cpu())
    p.check()


def test_on_another_stream():
    p = Pool(seqs=3, pages=20, most=8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        p.extend([0], [20])
        p.fork([0], [1])
        p.extend([1], [5], stream=side)
    side.synchronize()
    p.check()


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_pages_past_32_bits(fp8):
    """The last pages of a pool of more than 2^32 elements."""
    n, H, P, D = 70000, 8, 64, 128
    k, v = (torch.empty(1, n, H, P, D, dtype=U8 if fp8 else BF16, device="cuda") for _ in "kv")
    sc = [torch.empty(1, n, H, P, device="cuda") for _ in "kv"] if fp8 else [None, None]
    pages = fsx.Pages(k, v, 3, n, *sc)
    pages.extend([0, 1], [(n - 4) * P, P + 3])
    pages.fork([1], [2])
    g = torch.Generator().manual_seed(1)
    x = [torch.randn(1, 3, H, D, generator=g).to(BF16) for _ in "kv"]
    pages.extend([1], [3])
    pages.write(0, 1, x[0].cuda(), x[1].cuda(), [1], fsx.PackedRows([3]))
    table, length = pages.tables()
    assert length.tolist() == [(n - 4) * P, P + 6, P + 3] and table[1, 1] == n - 2
    for t, s, rows in zip((k, v), sc, x):
        got = t[0, n - 2, :, 3:6].transpose(0, 1).cpu()
        if fp8:
            code, scale = encode(rows[0])
            assert torch.equal(got, code) and torch.equal(s[0, n - 2, :, 3:6].t().cpu(), scale)
        else:
            assert torch.equal(got, rows[0])
    pages.keep([1], [[(P + 3, 3)]])
    assert pages.tables()[0][1, 0] == n - 1  # its first page is shared
    for t, rows in zip((k, v), x):
        got = t[0, n - 1, :, :3].transpose(0, 1).cpu()
        assert torch.equal(got, encode(rows[0])[0] if fp8 else rows[0])


def test_refusals():
    p = Pool(seqs=4, pages=10, most=5)
    p.extend([0], [20])
    p.fork([0], [1])
    k, v = (t.cuda() for t in p.new(20))

    def write(seqs, lens, layer=0, n=2, starts=None, k=k, v=v):
        p.pages.write(layer, n, k, v, seqs, fsx.PackedRows(lens, starts))

    for call, code, word in (
            (lambda: write([0], [1]), 1, "another sequence"), (lambda: write([1], [20]), 1, "another sequence"),
            (lambda: write([0], [21]), 1, "20 rows"), (lambda: write([2], [1]), 1, "0 rows"), (lambda: write([0, 0], [0, 0]), 1, "twice"),
            (lambda: write([4], [0]), 1, "max_seqs"), (lambda: write([0], [0], layer=1), 1, "layers"), (lambda: write([0], [0], layer=-1), 1, "layers"),
            (lambda: write([0], [4], starts=[17]), 1, "packed rows"), (lambda: write([0], [-1]), 1, "rows"),
            (lambda: p.pages.extend([0], [61]), 3, "pages"), (lambda: p.pages.extend([0, 1, 2, 3], [60, 60, 60, 1]), 3, "free"),
            (lambda: p.pages.extend([0] * 5, [1] * 5), 1, "n must"), (lambda: p.pages.keep([0], [[(0, 1)] * 257]), 2, "256 ranges"),
            (lambda: p.pages.keep([0], [[(0, 21)]]), 1, "ascend"), (lambda: p.pages.fork([0], [1]), 1, "has rows")):
        with pytest.raises(fsx.FsxError, match=word) as e:
            call()
        assert e.value.code == code
        p.check()
    for bad in (lambda: p.pages.write(0, 2, k.cpu(), v.cpu(), [0], fsx.PackedRows([0])), lambda: p.pages.write(0, 1, k, v, [0], fsx.PackedRows([0])),
                lambda: p.pages.write(0, 2, k, v[:, :5], [0], fsx.PackedRows([0])), lambda: p.pages.write(0, 2, k, v, [0, 1], fsx.PackedRows([0])),
                lambda: p.pages.extend([0], [1, 2]), lambda: p.pages.fork([0], [2, 3]), lambda: p.pages.keep([0], []),
                lambda: p.pages.extend([2 ** 31], [1])):
        with pytest.raises(ValueError):
            bad()
    write([0], [0])  # nothing to do
    p.pages.extend([], [])
    for bad in (lambda: fsx.Pages(p.k, p.v[:1], 1, 1), lambda: fsx.Pages(p.k, p.v, 1, 1, p.k, p.k), lambda: fsx.Pages(p.k.float(), p.v.float(), 1, 1, None),
                lambda: fsx.Pages(p.k.transpose(1, 2), p.v.transpose(1, 2), 1, 1), lambda: fsx.Pages(p.k.to(U8), p.v.to(U8), 1, 1),
                lambda: fsx.Pages(p.k.to(torch.int8), p.v.to(torch.int8), 1, 1), lambda: fsx.Pages(p.k.cpu(), p.v.cpu(), 1, 1)):
        with pytest.raises((ValueError, fsx.FsxError)):
            bad()
    within = p.k.view(2, -1, 2, 128)[:, 5:25]  # rows of the pool itself
    with pytest.raises(fsx.FsxError, match="pool"):
        p.pages.extend([2], [4])
        write([2], [4], k=within, v=v)
    p.free([2])
    odd = torch.randn(2, 20, 2, 132).to(BF16).cuda()[..., :128]
    with pytest.raises(fsx.FsxError, match="multiples of 8"):
        write([0], [0], k=odd, v=odd)
    p.check()
