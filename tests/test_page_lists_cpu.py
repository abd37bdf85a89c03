"""The host's lists of pages (csrc/page_lists.h) on the CPU: what a call reports is carried out on arrays that stand for the device's
lists and pool, where every row holds a name of its own, and compared with sequences kept as plain lists of those names."""

import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include <cstring>
#include "page_lists.h"
using namespace fsx;
extern "C" {
PageLists* make(int pages, int seqs, int most, int P) { return new PageLists(pages, seqs, most, P); }
void drop(PageLists* l) { delete l; }
int extend(PageLists* l, int n, const int* s, const int* r) { return l->extend(n, s, r); }
int fork_(PageLists* l, int n, const int* s, const int* d, const int* r) { return l->fork(n, s, d, r); }
int free_(PageLists* l, int n, const int* s) { return l->free(n, s); }
int keep(PageLists* l, int n, const int* s, const int* k, const int* f, const int* c) { return l->keep(n, s, k, f, c); }
int writable(PageLists* l, int s, int rows) { return l->writable(s, rows); }
const char* error(PageLists* l) { return l->error.c_str(); }
long n_free(PageLists* l) { return l->n_free; }
const int* data(PageLists* l, int what, int* n) {
  const std::vector<int32_t>* v = what == 0 ? &l->table : what == 1 ? &l->len : &l->ref;
  if (what < 3) { *n = (int)v->size(); return v->data(); }
  switch (what) {
    case 3: *n = 5 * (int)l->runs.size(); return (const int*)l->runs.data();
    case 4: *n = 5 * (int)l->before.size(); return (const int*)l->before.data();
    case 5: *n = 3 * (int)l->copies.size(); return (const int*)l->copies.data();
    case 6: *n = 2 * (int)l->ranges.size(); return (const int*)l->ranges.data();
    default: *n = 5 * (int)l->moves.size(); return (const int*)l->moves.data();
  }
}
}
"""
TABLE, LEN, REF, RUNS, BEFORE, COPIES, RANGES, MOVES = range(8)
OK, BAD, FULL = 0, 1, 3


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    at = tmp_path_factory.mktemp("lists")
    (at / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2607_15621_amd", "csrc"), str(at / "shim.cpp"), "-o", str(at / "shim.so")], check=True)
    L = ctypes.CDLL(str(at / "shim.so"))
    L.make.restype = ctypes.c_void_p
    L.data.restype = ctypes.POINTER(ctypes.c_int)
    L.error.restype = ctypes.c_char_p
    L.n_free.restype = ctypes.c_long
    return L


def ints(v):
    return (ctypes.c_int * max(1, len(v)))(*v)


class Lists:
    def __init__(self, L, pages, seqs, most, P):
        self.L, self.h, self.P, self.seqs = L, ctypes.c_void_p(L.make(pages, seqs, most, P)), P, seqs
        self.pool = np.full((pages, P), -1, np.int64)  # the device: names of rows, lists, lengths
        self.table, self.next, self.len = (np.full((seqs, most), -7), np.full((seqs, most), -8), np.zeros(seqs, np.int64))
        self.rows = [[] for _ in range(seqs)]          # what the sequences hold
        self.names = 0

    def __del__(self):
        self.L.drop(self.h)

    def data(self, what, width=1):
        n = ctypes.c_int()
        p = self.L.data(self.h, what, ctypes.byref(n))
        return np.array(p[:n.value], np.int64).reshape(-1, width)

    def apply(self, runs, table, lengths):
        old = self.table.copy()
        for s, at, first, count, length in runs:
            table[s, at:at + count] = old[~first, at:at + count] if first < 0 else np.arange(first, first + count)
            if lengths:
                self.len[s] = length

    def check(self):
        host, length, ref = self.data(TABLE).reshape(self.table.shape), self.data(LEN).ravel(), self.data(REF).ravel()
        used = np.zeros(len(ref), np.int64)
        for s in range(self.seqs):
            n = -(-len(self.rows[s]) // self.P)
            assert length[s] == self.len[s] == len(self.rows[s])
            assert (host[s, :n] == self.table[s, :n]).all() and (host[s, n:] == -1).all()
            np.add.at(used, host[s, :n], 1)
            got = self.pool[self.table[s, :n]].ravel()[:len(self.rows[s])]
            assert got.tolist() == self.rows[s], s
        assert (used == ref).all() and self.L.n_free(self.h) == int((used == 0).sum())

    def extend(self, seqs, rows, want=OK):
        assert self.L.extend(self.h, len(seqs), ints(seqs), ints(rows)) == want, self.L.error(self.h)
        if want != OK:
            return self.check()
        for a, b, n in self.data(COPIES, 3):
            self.pool[b, :n] = self.pool[a, :n]
        self.apply(self.data(RUNS, 5), self.table, True)
        for s, n in zip(seqs, rows):  # written as they would be
            assert self.L.writable(self.h, s, n)
            for _ in range(n):
                i = len(self.rows[s])
                self.pool[self.table[s, i // self.P], i % self.P] = self.names
                self.rows[s].append(self.names)
                self.names += 1
        self.check()

    def fork(self, src, dst, rows=None, want=OK):
        assert self.L.fork_(self.h, len(src), ints(src), ints(dst), ints(rows) if rows is not None else None) == want, self.L.error(self.h)
        if want == OK:
            self.apply(self.data(RUNS, 5), self.table, True)
            for i, (a, b) in enumerate(zip(src, dst)):
                self.rows[b] = self.rows[a][:rows[i] if rows is not None else None]
        self.check()

    def free(self, seqs, want=OK):
        assert self.L.free_(self.h, len(seqs), ints(seqs)) == want, self.L.error(self.h)
        if want == OK:
            self.apply(self.data(RUNS, 5), self.table, True)
            for s in seqs:
                self.rows[s] = []
        self.check()

    def keep(self, seqs, ranges, want=OK):
        flat = [x for r in ranges for x in r]
        assert self.L.keep(self.h, len(seqs), ints(seqs), ints([len(r) for r in ranges]), ints([a for a, _ in flat]),
                           ints([n for _, n in flat])) == want, self.L.error(self.h)
        if want != OK:
            return self.check()
        before, spans = self.data(BEFORE, 5), self.data(RANGES, 2)
        self.apply(before, self.next, False)
        to = self.next if len(before) else self.table
        moves = self.data(MOVES, 5).tolist()
        random.Random(self.names).shuffle(moves)  # the workgroups of different sequences run in any order, stretch by stretch
        at = {m[0]: m[3] for m in moves}
        while moves:
            m = moves[self.names % len(moves)]
            s, first, n, start, rows = m
            source = [r for a, c in spans[first:first + n] for r in range(a, a + c)]
            assert len(source) == rows
            i0 = at[s]
            i1 = min(rows, i0 + 5)
            x = [self.pool[self.table[s, r // self.P], r % self.P] for r in source[i0:i1]]
            for i in range(i0, i1):
                self.pool[to[s, i // self.P], i % self.P] = x[i - i0]
            at[s] = i1
            self.names += 1
            if i1 == rows:
                moves.remove(m)
        self.apply(self.data(RUNS, 5), self.table, True)
        for s, r in zip(seqs, ranges):
            self.rows[s] = [x for a, n in r for x in self.rows[s][a:a + n]]
        self.check()


def test_a_fork_shares_and_the_last_sharer_keeps(lib):
    l = Lists(lib, 6, 4, 4, 16)
    l.extend([0], [20])
    l.fork([0, 0], [1, 2])
    assert lib.n_free(l.h) == 4 and not lib.writable(l.h, 0, 1)
    l.extend([2, 1], [1, 13])  # 2 copies, 1 copies (0 still has the page), and takes a third
    assert l.data(TABLE).reshape(4, 4)[:3].tolist() == [[0, 1, -1, -1], [0, 3, 4, -1], [0, 2, -1, -1]]
    l.free([0])  # page 1 alone becomes free
    l.extend([1], [0])
    assert lib.n_free(l.h) == 2 and lib.writable(l.h, 1, 17) and not lib.writable(l.h, 1, 18)
    l.fork([1], [3], [17])
    l.extend([1, 3], [15, 1])  # 1 fills its own third page; 3 copies one row of the second
    assert l.data(COPIES, 3).tolist() == [[3, 1, 1]]


def test_sharers_named_in_one_call(lib):
    l = Lists(lib, 4, 2, 4, 16)
    l.extend([0], [5])
    l.fork([0], [1])
    l.extend([0, 1], [1, 1])
    assert l.data(TABLE).reshape(2, 4)[:, 0].tolist() == [1, 0]
    assert l.data(COPIES, 3).tolist() == [[0, 1, 5]]


def test_errors_change_nothing(lib):
    l = Lists(lib, 4, 4, 3, 16)
    l.extend([0, 1], [20, 3])
    l.fork([1], [3])
    l.extend([0], [29], FULL)         # past its three pages
    l.extend([0, 2], [13, 16], FULL)  # two pages, one is free
    l.extend([1, 3, 0], [1, 1, 13], FULL)
    l.extend([0, 0], [1, 1], BAD)
    l.extend([4], [1], BAD)
    l.extend([-1], [1], BAD)
    l.extend([0], [-1], BAD)
    l.fork([0], [1], want=BAD)
    l.fork([0, 0], [2, 2], want=BAD)
    l.fork([0], [0], want=BAD)
    l.fork([0, 2], [2, 3], want=BAD)
    l.fork([4], [2], want=BAD)
    l.fork([0], [2], [21], want=BAD)
    l.fork([0], [2], [-1], want=BAD)
    l.free([1, 1], BAD)
    l.free([9], BAD)
    l.keep([0], [[(0, 21)]], BAD)
    l.keep([0], [[(5, 3), (7, 2)]], BAD)
    l.keep([0], [[(5, -1)]], BAD)
    l.keep([0], [[(-1, 2)]], BAD)
    l.extend([1, 3], [1, 1])  # one copy takes the last page
    l.fork([0], [2])
    l.keep([2], [[(1, 19)]], FULL)  # both pages are shared


@pytest.mark.parametrize("seed", range(40))
def test_random_calls(lib, seed):
    r = random.Random(seed)
    P = r.choice([16, 32])
    seqs, most = r.choice([2, 5, 9]), r.choice([2, 4, 9])
    l = Lists(lib, r.choice([8, 30, 70, 130]), seqs, most, P)

    def full(call, *args):
        """The call, whichever of a result and too few pages it should give."""
        need = want(*args)
        call(*args, OK if need <= lib.n_free(l.h) else FULL)

    for _ in range(60):
        some = r.sample(range(seqs), r.randint(1, seqs))
        what = r.choice(["extend"] * 4 + ["fork"] * 2 + ["keep"] * 3 + ["free"])
        if what == "extend":
            rows = [r.choice([0, 1, 1, 5, P, 3 * P]) for _ in some]
            rows = [min(n, most * P - len(l.rows[s])) for s, n in zip(some, rows)]

            def want(some, rows):
                ref, need = l.data(REF).ravel().copy(), 0
                for s, n in zip(some, rows):
                    have, at = -(-len(l.rows[s]) // P), len(l.rows[s])
                    need += -(-(at + n) // P) - have
                    if n and at % P and ref[l.table[s, have - 1]] > 1:
                        ref[l.table[s, have - 1]] -= 1
                        need += 1
                return need
            full(l.extend, some, rows)
        elif what == "fork":
            dst = [s for s in some if not l.rows[s]]
            src = [s for s in range(seqs) if s not in dst]
            if dst and src:
                src = [r.choice(src) for _ in dst]
                l.fork(src, dst, [r.randint(0, len(l.rows[s])) for s in src] if r.random() < 0.5 else None)
        elif what == "free":
            l.free(some)
        else:
            ranges = []
            for s in some:
                cut = sorted(r.randint(0, len(l.rows[s])) for _ in range(2 * r.choice([0, 1, 1, 2, 5])))
                ranges.append([(a, b - a) for a, b in zip(cut[::2], cut[1::2])])

            def want(some, ranges):
                ref, need = l.data(REF).ravel(), 0
                for s, x in zip(some, ranges):
                    source = [i for a, n in x for i in range(a, a + n)]
                    moved = [i for i, j in enumerate(source) if i != j]
                    if moved:
                        need += sum(ref[l.table[s, j]] > 1 for j in range(moved[0] // P, -(-len(source) // P)))
                return need
            full(l.keep, some, ranges)
