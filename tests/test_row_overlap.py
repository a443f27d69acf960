"""Which rows share memory (csrc/row_overlap.cuh, compiled for the host) against sets of all their places."""
import ctypes
import random
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2011_09398_b200" / "csrc"
SOURCE = """
#include "row_overlap.cuh"
using namespace lce;
static RowSet set(const int64_t *s) { return {(const void *)s[0], s[1], s[2], s[3], s[4], s[5], s[6]}; }
extern "C" int apart(const int64_t *a) { return rows_apart(set(a)); }
extern "C" int meet(const int64_t *a, const int64_t *b) { return rows_meet(set(a), set(b)); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    where = tmp_path_factory.mktemp("row_overlap")
    (where / "rows.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", "-o", str(where / "rows.so"), str(where / "rows.cpp")], check=True)
    return ctypes.CDLL(str(where / "rows.so"))


def array(s):
    return (ctypes.c_int64 * 7)(*s)


def rows(s):
    data, outer, inner, outer_stride, inner_stride, length, size = s
    return [set(range(data + (i * outer_stride + j * inner_stride) * size, data + (i * outer_stride + j * inner_stride + length) * size)) for i in range(outer) for j in range(inner)]


def draw(rng, size):
    return [4096 + 4 * rng.randint(0, 40), rng.randint(0, 4) or 1, rng.randint(0, 4) or 1, rng.choice([0, 1, 2, 5, 8, 13, 16, 24, 40]), rng.choice([0, 1, 2, 3, 4, 5, 8, 12, 20]),
            rng.randint(0, 6), size]


def test_rows_apart(lib):
    rng, answers = random.Random(1), []
    for _ in range(4000):
        s = draw(rng, rng.choice([2, 4]))
        all_rows = rows(s)
        answers.append(len(set().union(*all_rows)) == sum(map(len, all_rows)))
        assert bool(lib.apart(array(s))) == answers[-1], s
    assert 500 < sum(answers) < 3500


def test_rows_meet(lib):
    rng, answers = random.Random(2), []
    for _ in range(6000):
        size = rng.choice([2, 4])
        a, b = draw(rng, size), draw(rng, size)
        if rng.random() < 0.7:
            b[3] = a[3]  # the same outer stride, as views into one buffer have it
        if rng.random() < 0.5:
            b[4] = a[4]
        want = bool(set().union(*rows(a)) & set().union(*rows(b)))
        got = bool(lib.meet(array(a), array(b)))
        assert got == bool(lib.meet(array(b), array(a)))
        answers.append(want)
        assert got == want, (a, b)
    assert 1000 < sum(answers) < len(answers) - 1000


def test_large_numbers(lib):
    most = (1 << 40) - 1
    assert lib.apart(array([4096, 1 << 31, 65535, most, 16, 8, 4]))
    assert not lib.apart(array([4096, 1 << 31, 65535, 16, most, 17, 4]))
    assert not lib.meet(array([1 << 45, 1 << 31, 65535, most, most, 256, 4]), array([4096, 1, 1, 0, 0, 256, 4]))
    # queries and keys side by side in rows of one buffer, turned in place
    q, k = [4096, 1 << 30, 32, 6144, 128, 128, 2], [4096 + 2 * 4096, 1 << 30, 8, 6144, 128, 128, 2]
    assert not lib.meet(array(q), array(k)) and lib.meet(array(q), array([k[0] - 2, *k[1:]]))
    assert lib.meet(array(q), array([4096 + 2 * 6144 * ((1 << 30) - 1), 1, 1, 0, 0, 1, 2])) and not lib.meet(array(q), array([4096 + 2 * (6144 * 9 + 4096), 1, 1, 0, 0, 2048, 2]))
