"""What the calls of the pages write, and nothing else: after every call all four tensors of the pool are compared bit for bit with
what they held before it, outside the rows that sequences have, which hold what they should (codes and scales included)."""

from __future__ import annotations

import numpy as np
import pytest
import torch

from gpu_pages import BF16, F32, U8, Pool
from paper_2607_15621_amd import fsx

pytestmark = pytest.mark.gpu

kinds = pytest.mark.parametrize("fp8,D", [(False, 128), (False, 64), (True, 128), (True, 64)], ids=["bf16-128", "bf16-64", "fp8-128", "fp8-64"])


class WatchedPool(Pool):
    """A pool of random bits that looks at itself after every call.  No call has a reason to write a row that no sequence has when it
    returns: copies, moved rows and new ones all belong to a sequence then."""

    def __init__(self, **kw):
        super().__init__(**kw)
        g = torch.Generator(device="cuda").manual_seed(17)
        self.tensors = [t for t in (self.k, self.v, self.ks, self.vs) if t is not None]
        for t in self.tensors:
            b = t.view(U8)
            b.copy_(torch.randint(0, 256, b.shape, generator=g, device="cuda", dtype=torch.int32).to(U8))
        self.look()

    def look(self):
        self.seen = [t.view(U8).clone() for t in self.tensors]

    def check(self):
        super().check()
        table, length = self.pages.tables()
        had = torch.zeros(self.k.shape[1], self.P, dtype=torch.bool)
        for s in range(self.seqs):
            for i in range(int(length[s])):
                had[table[s, i // self.P], i % self.P] = True
        for t, b in zip(self.tensors, self.seen):
            differs = t.view(U8) != b
            # [layers][pages][heads][rows][bytes]: of codes a byte each, of scales four to a row
            differs = differs.reshape(*t.shape[:3], self.P, -1).any(4).any(2).any(0).cpu()
            assert not bool((differs & ~had).any()), (differs & ~had).nonzero()[:8]
        self.look()

    def extend(self, seqs, counts, dtype=BF16, write=True, stream=None):
        self.pages.extend(seqs, counts, stream=stream)
        grown = [list(self.rows[s]) for s in seqs]
        table, _ = self.pages.tables()
        k, v = self.new(sum(counts), dtype)
        # rows with room and no contents yet hold what lies there (of a copied page: what was not copied)
        host = [t.cpu() for t in self.tensors]
        for s, n in zip(seqs, counts):
            at = len(self.rows[s])
            for i in range(at, at + n):
                page, r = int(table[s, i // self.P]), i % self.P
                self.rows[s].append(tuple(t[:, page, :, r].clone() for t in host))
        self.check()
        self.pages.write(0, self.L, k.cuda(), v.cuda(), seqs, fsx.PackedRows(counts), stream=stream)
        at, stored = 0, self.stored(k, v)
        for s, n, rows in zip(seqs, counts, grown):
            self.rows[s] = rows + stored[at:at + n]
            at += n
        self.check()

    def fork(self, *a):
        super().fork(*a)
        self.check()

    def keep(self, *a):
        super().keep(*a)
        self.check()

    def free(self, *a):
        super().free(*a)
        self.check()


def test_a_stray_byte_is_seen():
    """The watch itself: a byte behind a sequence's end, in a free page, in a stale scale."""
    p = WatchedPool(seqs=2, pages=6, most=3, fp8=True)
    p.extend([0], [19])
    table, _ = p.pages.tables()
    for t, at in ((p.k, (1, table[0, 1], 0, 3, 5)), (p.v, (0, 5, 1, 0, 127)), (p.ks, (0, table[0, 1], 1, 15)), (p.vs, (1, 4, 0, 0))):
        was = t[at].item()
        t[at] = (was + 1) % 128 if t.dtype is U8 else 0.25
        with pytest.raises(AssertionError):
            p.check()
        p.look()


@kinds
@pytest.mark.parametrize("P", [16, 64, 256])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["from-bf16", "from-f32"])
def test_rows_written(fp8, D, P, dtype):
    p = WatchedPool(pages=24, seqs=6, most=8, P=P, D=D, fp8=fp8)
    p.extend([0, 3, 5, 1], [1, P, P + 1, 5], dtype)
    p.extend([5, 0, 3], [P - 1, 1, 2 * P], dtype)
    p.extend([2], [0], dtype)


@kinds
@pytest.mark.parametrize("P", [16, 128])
def test_forks_diverge(fp8, D, P):
    p = WatchedPool(pages=40, seqs=8, most=6, P=P, D=D, fp8=fp8)
    p.extend([0], [2 * P + 5])
    p.fork([0] * 5, [1, 2, 3, 4, 5])
    p.extend([1, 2], [1, P])
    p.extend([0, 3, 4, 5], [1, 2, 3, 4])
    p.fork([1, 1], [6, 7], [P + 3, 2])
    p.extend([6, 7, 1], [2, 2, 2])


@kinds
@pytest.mark.parametrize("ranges", [[(0, 50)], [(0, 16), (32, 60)], [(1, 91)], [(3, 5), (20, 1), (21, 4), (40, 52)], [(0, 0)], [(91, 1)], [],
                                    [(i, 1) for i in range(0, 92, 3)]], ids=str)
def test_rows_kept(fp8, D, ranges):
    p = WatchedPool(pages=40, seqs=5, most=8, P=16, D=D, fp8=fp8)
    p.extend([0, 1, 2], [92, 92, 92])
    p.fork([1], [3])
    p.fork([2], [4], [40])
    p.keep([0, 1, 2], [ranges] * 3)
    p.free([1])
    p.keep([3], [ranges])


@pytest.mark.parametrize("seed", range(8))
def test_random_calls(seed):
    rng = np.random.default_rng(100 + seed)
    fp8, P = bool(seed % 2), [16, 32, 64, 128][seed // 2]
    p = WatchedPool(pages=30, seqs=7, most=6, P=P, D=[128, 64][seed % 3 == 0], fp8=fp8, L=1 + seed % 2, H=1 + seed % 3)
    for _ in range(24):
        some = [int(s) for s in rng.permutation(7)[:rng.integers(1, 4)]]
        what = rng.integers(0, 5)
        before = [list(r) for r in p.rows]
        try:
            if what <= 1:
                p.extend(some, [int(x) for x in rng.integers(0, 2 * P, len(some))], [BF16, F32][seed % 2])
            elif what == 2:
                empty = [s for s in range(7) if not p.rows[s]]
                full = [s for s in range(7) if p.rows[s]]
                if not empty or not full:
                    continue
                dst = empty[:2]
                src = [int(x) for x in rng.choice(full, len(dst))]
                p.fork(src, dst, [int(rng.integers(0, len(p.rows[s]) + 1)) for s in src])
            elif what == 3:
                ranges = []
                for s in some:
                    cuts = sorted(int(x) for x in rng.integers(0, len(p.rows[s]) + 1, 4))
                    ranges.append([(cuts[0], cuts[1] - cuts[0]), (cuts[2], cuts[3] - cuts[2])])
                p.keep(some, ranges)
            else:
                p.free(some[:2])
        except fsx.FsxError as e:
            assert e.code == 3  # too few pages, or a sequence at its most: nothing changed
            p.rows = before
            p.check()
