"""Which rows share memory, against sets of bytes (compiled from the header that the binding includes; nothing here needs a GPU)."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2104_14129_amd import build

HARNESS = '''
#include "actq_overlap.h"
using namespace actq;
static Strips of(const int64_t* v) { return strips_of(v[0], v[1], v[2], v[3], v[4], v[5]); }
extern "C" {
int strips(const int64_t* a, const int64_t* b) { return overlap({a[0], a[2], a[1], a[5]}, Strip{b[0], b[2], b[1], b[5]}); }
int tensors(const int64_t* a, const int64_t* b) { return overlap(of(a), of(b)); }
int separate(const int64_t* a) { return apart(of(a)); }
}
'''


@pytest.fixture(scope="module")
def library(tmp_path_factory):
    at = tmp_path_factory.mktemp("overlap")
    (at / "harness.cpp").write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fPIC", "-shared", "-I", build.CSRC, "-o", str(at / "harness.so"), str(at / "harness.cpp")], check=True)
    return ctypes.CDLL(os.path.join(at, "harness.so"))


def _call(f, *tensors):
    return bool(f(*[(ctypes.c_int64 * 6)(*t) for t in tensors]))


def _bytes(first, rows, stride, heads, head_stride, size):
    return [first + r * stride + h * head_stride + i for r in range(rows) for h in range(heads) for i in range(size)]


def test_rows(library):
    """Of every kind: expanded, next to each other, apart, backwards, none; at equal and other strides."""
    rng = random.Random(1)
    seen = [0, 0]
    for _ in range(40000):
        a, b = ([rng.randrange(60), rng.randrange(6), rng.choice([rng.randrange(-20, 21), 12]), 1, 0, rng.randrange(8)] for _ in range(2))
        if rng.random() < 0.5:
            b[2] = a[2]
        want = bool(set(_bytes(*a)) & set(_bytes(*b)))
        seen[want] += 1
        assert _call(library.strips, a, b) == _call(library.strips, b, a) == want, (a, b)
    assert min(seen) > 5000


def test_tensors_of_heads(library):
    rng = random.Random(2)
    seen = [0, 0]
    for _ in range(40000):
        size = rng.randrange(1, 6)
        strides = [0, size, size * 2, size * 3, size * 6, rng.randrange(40)]
        a, b = ([rng.randrange(100), rng.randrange(4), rng.choice(strides), rng.randrange(4), rng.choice(strides), size] for _ in range(2))
        if rng.random() < 0.3:
            b = list(a)
        mine, other = _bytes(*a), _bytes(*b)
        want = bool(set(mine) & set(other))
        seen[want] += 1
        assert _call(library.tensors, a, b) == _call(library.tensors, b, a) == want, (a, b)
        assert _call(library.separate, a) == (len(set(mine)) == len(mine)), a
    assert min(seen) > 5000


def test_far_apart_and_long(library):
    """Offsets beyond 32 bits; columns of a wide matrix by turns; a single shared byte at the end."""
    wide, rows = 1 << 21, 1 << 20
    left, right = [0, rows, wide, 1, 0, wide // 2], [wide // 2, rows, wide, 1, 0, wide // 2]
    assert not _call(library.strips, left, right)
    assert _call(library.strips, left, [wide // 2 - 1, rows, wide, 1, 0, 1])
    assert _call(library.strips, left, [(rows - 1) * wide + wide // 2 - 1, 1, 0, 1, 0, 1])
    assert not _call(library.strips, left, [(rows - 1) * wide + wide // 2, 1, 0, 1, 0, 1])
    assert not _call(library.strips, [0, rows, 2 * wide, 1, 0, wide], [wide, rows, 2 * wide, 1, 0, wide])   # every other row
    assert not _call(library.strips, [0, 1000, 4 * wide, 1, 0, wide], [wide, 2000, 2 * wide, 1, 0, wide])
    assert _call(library.strips, [0, 1000, 4 * wide, 1, 0, wide], [wide, 2000, 3 * wide, 1, 0, wide])
