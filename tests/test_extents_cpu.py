"""Rows and heads of tensors that overlap (csrc/extents.h), on the CPU, against sets of bytes."""

import ctypes
import itertools
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHIM = r"""
#include "extents.h"
using namespace fsx;
extern "C" {
int apart_(const int64_t* x) { return apart({x[0], x[1], x[2], x[3], x[4], x[5]}); }
int meet_(const int64_t* a, const int64_t* b) { return meet({a[0], a[1], a[2], a[3], a[4], a[5]}, {b[0], b[1], b[2], b[3], b[4], b[5]}); }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    at = tmp_path_factory.mktemp("extents")
    (at / "shim.cpp").write_text(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2607_15621_amd", "csrc"), str(at / "shim.cpp"), "-o", str(at / "shim.so")], check=True)
    return ctypes.CDLL(str(at / "shim.so"))


def six(x):
    return (ctypes.c_int64 * 6)(*x)


def runs(x):
    at, rows, row, heads, head, dim = x
    return [(at + r * row + h * head, at + r * row + h * head + dim) for r, h in itertools.product(range(rows), range(heads))]


def covered(x):
    return {b for a, e in runs(x) for b in range(a, e)}


def overlaps_itself(x):
    """As the library takes it: runs that share a byte, or blocks of one stride's runs that reach into each other."""
    return len(covered(x)) < x[1] * x[3] * x[5]


@pytest.mark.parametrize("seed", range(8))
def test_random(lib, seed):
    rng = random.Random(seed)
    hit = nested = 0
    for _ in range(6000):
        def extent():
            dim = rng.choice([1, 2, 4, 8])
            rows, heads = rng.randint(1, 5), rng.randint(1, 5)
            if rng.random() < 0.7:  # one stride over the other, gaps between
                lo = dim * rng.choice([1, 1, 2, 3])
                inner = rng.randint(1, 5)
                hi = (inner - 1) * lo + dim + rng.choice([0, 0, 1, 2, 7, 16, 40])
                outer = rng.randint(1, 5)
                return (rng.randint(0, 150), outer, hi, inner, lo, dim) if rng.random() < 0.5 else (rng.randint(0, 150), inner, lo, outer, hi, dim)
            return rng.randint(0, 150), rows, rng.choice([0, rng.randint(0, 40)]), heads, rng.choice([0, rng.randint(0, 40)]), dim
        a, b = extent(), extent()
        if rng.random() < 0.4 and b[2]:  # rows of one length
            a = (a[0], a[1], b[2], *a[3:])
        if lib.apart_(six(a)):
            assert not overlaps_itself(a), a
        if not lib.apart_(six(b)):
            continue
        assert not overlaps_itself(b), b
        want = bool(covered(a) & covered(b))
        assert bool(lib.meet_(six(a), six(b))) == want, (a, b)
        hit += want
        nested += not want and a[0] < max(e for _, e in runs(b)) and b[0] < max(e for _, e in runs(a))
    assert hit > 500 and nested > 50


def test_heads_side_by_side_in_a_row(lib):
    """Sixteen rows of 32 + 8 + 8 heads of 256 bytes: parts of the rows do not meet, the same heads do, heads that begin within do."""
    row, head = 48 * 256, 256
    q, k = (0, 16, row, 32, head, 256), (32 * 256, 16, row, 8, head, 256)
    assert lib.apart_(six(q)) and lib.apart_(six(k))
    assert not lib.meet_(six(q), six(k)) and not lib.meet_(six(k), six(q))
    assert lib.meet_(six(q), six(q)) and lib.meet_(six(q), six((31 * 256, 16, row, 8, head, 256)))
    assert lib.meet_(six(q), six((31 * 256 + 255, 16, row, 1, head, 256))) and not lib.meet_(six(q), six((-256, 16, row, 1, head, 256)))
    assert lib.meet_(six(q), six((-255, 16, row, 1, head, 256)))
    # heads in turn: every second one
    even, odd = (0, 16, row, 24, 512, 256), (256, 16, row, 24, 512, 256)
    assert not lib.meet_(six(even), six(odd)) and lib.meet_(six(even), six((255, 16, row, 24, 512, 256)))


def test_the_largest(lib):
    """Offsets far past 32 bits; a step for every run would take minutes."""
    row = 2 * 4096 * 512 * 16
    a, b = (1 << 40, 65536, row, 4096, 512, 512), ((1 << 40) + 4096 * 512, 65536, row, 4096, 512, 512)
    assert not lib.meet_(six(a), six(b)) and lib.meet_(six(a), six(((1 << 40) + 4096 * 512 - 1, 65536, row, 1, 0, 512)))
    assert lib.meet_(six((0, 1, 0, 1, 0, 1 << 56)), six(b)) and not lib.meet_(six((0, 1, 0, 1, 0, 1 << 40)), six(b))
