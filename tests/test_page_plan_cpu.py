"""How the attention over pages is shared out (plan_page_attention of the built library), on the CPU."""

import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include "kernels.h"
using namespace fsx;
extern "C" {
PageLists* make(int pages, int seqs, int most, int P) { return new PageLists(pages, seqs, most, P); }
void drop(PageLists* l) { delete l; }
int extend(PageLists* l, int n, const int* s, const int* r) { return l->extend(n, s, r); }
int fork_(PageLists* l, int n, const int* s, const int* d, const int* r) { return l->fork(n, s, d, r); }
// launches: first, n, first_tile, n_tiles, per, each, extra, workgroups, parts; entries: index, base, steps, own, shared; tiles: first, members
long plan(PageLists* l, int Hk, int D, int fp8, int H, int n, const int* seqs, long bytes, int* launches, int* n_launches, int* entries,
          int* tiles, int* n_tiles, int* wide) {
  PagePool p{};
  p.Hk = Hk, p.P = l->P, p.D = D, p.fp8 = fp8, p.most = l->most, p.pages = l->n_pages, p.layers = 1;
  PagePlan plan;
  plan_page_attention(p, *l, H, n, seqs, bytes, plan);
  *n_launches = (int)plan.launches.size(), *n_tiles = (int)plan.tiles.size(), *wide = plan.wide;
  for (const auto& x : plan.launches)
    for (int v : {x.first, x.n, x.first_tile, x.n_tiles, x.per, x.each, x.extra, x.workgroups, x.parts}) *launches++ = v;
  for (const auto& x : plan.entries)
    for (int v : {x.index, x.base, x.steps, x.own, x.shared}) *entries++ = v;
  for (const auto& x : plan.tiles)
    for (int v : {x.first, x.members}) *tiles++ = v;
  return plan.bytes;
}
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    from paper_2607_15621_amd import build, fsx

    fsx.lib()
    at = tmp_path_factory.mktemp("plan")
    (at / "shim.hip").write_text(SHIM)
    subprocess.run([build.HIPCC, "-std=c++17", "-O1", "--offload-host-only", "-fPIC", "-I", build.CSRC, "-c", str(at / "shim.hip"), "-o", str(at / "shim.o")],
                   check=True, capture_output=True)
    subprocess.run(["g++", "-shared", str(at / "shim.o"), build.LIB, "-Wl,-rpath," + os.path.dirname(build.LIB), "-o", str(at / "shim.so")], check=True)
    L = ctypes.CDLL(str(at / "shim.so"))
    L.make.restype = ctypes.c_void_p
    L.plan.restype = ctypes.c_long
    return L


def ints(v):
    return (ctypes.c_int * max(1, len(v)))(*v)


UNBOUND = 2 ** 62


class Lists:
    def __init__(self, lib, lens, P=16, seqs=None):
        self.lib, self.P = lib, P
        self.h = ctypes.c_void_p(lib.make(sum(-(-n // P) for n in lens) + 1200, seqs or len(lens), max(1, max(-(-n // P) for n in lens)) + 40, P))
        assert lib.extend(self.h, len(lens), ints(range(len(lens))), ints(lens)) == 0

    def fork(self, src, dst, grow):
        assert self.lib.fork_(self.h, len(src), ints(src), ints(dst), None) == 0
        assert self.lib.extend(self.h, len(dst), ints(dst), ints(grow)) == 0

    def plan(self, seqs, Hk=8, G=4, D=128, fp8=False, workspace=UNBOUND):
        n = len(seqs)
        launches, entries, tiles, a, b, w = (ctypes.c_int * (9 * n))(), (ctypes.c_int * (5 * n))(), (ctypes.c_int * (2 * n + 2))(), *(ctypes.c_int() for _ in "abw")
        got = self.lib.plan(self.h, Hk, D, int(fp8), Hk * G, n, ints(seqs), ctypes.c_long(workspace), launches, ctypes.byref(a), entries, tiles,
                            ctypes.byref(b), ctypes.byref(w))
        names = ("first", "n", "first_tile", "n_tiles", "per", "each", "extra", "workgroups", "parts")
        return dict(bytes=got, wide=w.value, launches=[dict(zip(names, launches[9 * i:9 * i + 9])) for i in range(a.value)],
                    entries=[dict(zip(("index", "base", "steps", "own", "shared"), entries[5 * i:5 * i + 5])) for i in range(n)],
                    tiles=[tuple(tiles[2 * i:2 * i + 2]) for i in range(b.value)])

    def close(self):
        self.lib.drop(self.h)


def state(Hk, G, D):
    """Bytes of a part, all heads."""
    c = 16 if G <= 16 else 32
    return 4 * Hk * -(-G // c) * ((min(G, c) * (D + 2) + 3) // 4 * 4)


def bound(n, Hk, G, D):
    c = 16 if G <= 16 else 32
    t, w = (16 // G if G <= 8 else 1), max(1, 256 // (Hk * -(-G // c)))
    return state(Hk, G, D) * (2 * t * w * -(-n // 113) + 3 * n)


def check(p, s):
    """Parts are counted for the entries that are split, and no others."""
    total = 0
    for l in p["launches"]:
        split = [x["own"] + x["shared"] for x in p["entries"][l["first"]:l["first"] + l["n"]]]
        assert l["parts"] == sum(m for m in split if m > 1)
        assert l["workgroups"] >= 1
        total += l["parts"]
    assert p["bytes"] == total * s
    assert sorted(x["index"] for x in p["entries"]) == list(range(len(p["entries"])))


def test_one_part_too_few(lib):
    """64 long histories, 32 heads over 8: with a workspace one part short the shares stay even, over nearly as many workgroups."""
    l = Lists(lib, [501 + 229 * ((37 * i) % 64) for i in range(64)], 64)
    full = l.plan(range(64))
    s = state(8, 4, 128)
    check(full, s)
    assert full["launches"][0]["each"] == 0 and full["launches"][0]["workgroups"] == 32
    for short in range(1, 5):
        p = l.plan(range(64), workspace=full["bytes"] - s * short)
        check(p, s)
        assert p["bytes"] <= full["bytes"] - s * short
        assert p["launches"][0]["each"] == 0 and p["launches"][0]["workgroups"] >= 28
    l.close()


def test_entries_that_are_not_split_take_no_workspace(lib):
    """One history of 60,000 rows among 63 of 10."""
    l = Lists(lib, [60000] + [10] * 63)
    p = l.plan(range(64), Hk=32, G=1)
    check(p, state(32, 1, 128))
    long = [x for x in p["entries"] if x["index"] == 0][0]
    assert long["own"] > 4 and p["bytes"] == long["own"] * state(32, 1, 128)
    l.close()


@pytest.mark.parametrize("seed", range(30))
def test_any_workspace(lib, seed):
    """What is planned fits the workspace there is, down to none, and what would be planned without a limit the documented bound."""
    rng = random.Random(seed)
    n = rng.choice([1, 2, 5, 16, 33, 64, 130, 300])
    Hk, G, D, P = rng.choice([1, 2, 8, 32, 300]), rng.choice([1, 2, 3, 4, 5, 8, 9, 16, 20, 33]), rng.choice([64, 128]), rng.choice([16, 64])
    lens = [rng.choice([0, 1, rng.randint(2, 400), rng.randint(400, 9000)]) for _ in range(n)]
    base = rng.random() < 0.5
    if base:
        lens = [rng.randint(300, 4000)] * 2
    l = Lists(lib, lens, P, max(n, 2))
    if base and n > 2:
        l.fork([i % 2 for i in range(2, n)], list(range(2, n)), [rng.randint(0, 2 * P) if i % 3 else 0 for i in range(2, n)])
    seqs = list(range(n))
    if rng.random() < 0.3:
        seqs = [rng.randrange(n) for _ in range(n)]
    s = state(Hk, G, D)
    full = l.plan(seqs, Hk, G, D)
    check(full, s)
    assert full["bytes"] <= bound(n, Hk, G, D)
    for x in sorted({0, 1, s, 2 * s - 1, 2 * s, full["bytes"] // 9, full["bytes"] // 3, full["bytes"] // 2, full["bytes"] * 3 // 4, max(0, full["bytes"] - s),
                     max(0, full["bytes"] - 1)}):
        p = l.plan(seqs, Hk, G, D, workspace=x)
        check(p, s)
        assert p["bytes"] <= x or p["bytes"] == 0
    assert l.plan(seqs, Hk, G, D, workspace=full["bytes"]) == full
    l.close()
