"""The search for the k-th largest weight ends after three passes, also in a row that is
written while it is read (rows past the registers are read again in each pass), and finds
the k-th of one that is not (CPU)."""
import ctypes
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

from paper_2606_24506_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    out = str(tmp_path_factory.mktemp("search") / "shim.so")
    subprocess.run(["g++", "-std=c++17", "-O2", "-shared", "-fPIC", "-I", build.CSRC,
                    os.path.join(HERE, "c", "search_shim.cpp"), "-o", out], check=True)
    return ctypes.CDLL(out)


def search(lib, rows, k):
    """rows [passes][n]; the range is the first's."""
    rows = np.ascontiguousarray(rows, dtype=np.uint32)
    out = (ctypes.c_uint32 * 2)()
    lo, hi = int(rows[0].min()), int(rows[0].max())
    passes = lib.search(ctypes.c_void_p(rows.ctypes.data), rows.shape[0], rows.shape[1], k, lo, hi, out)
    return passes, out[0], out[1]


def draw(kind, n, rng):
    if kind == "any":
        return rng.integers(1, 1 << 32, n, dtype=np.uint64)
    if kind == "near":
        return (1 << 31) + rng.integers(0, 3000, n, dtype=np.uint64)
    if kind == "few":
        return rng.choice(np.array([1, 2, 1 << 31, (1 << 32) - 1], dtype=np.uint64), n)
    x = np.full(n, 1 << 31, dtype=np.uint64)  # mostly one
    x[rng.random(n) < 0.1] = 0xBF000000
    return x


@pytest.mark.parametrize("kind", ["any", "near", "few", "mostly"])
def test_the_kth_largest(lib, kind):
    rng = np.random.default_rng(1)
    for n in (2, 3, 100, 5000):
        for _ in range(60):
            row = draw(kind, n, rng)
            k = int(rng.integers(1, n))
            passes, key, equal = search(lib, row[None], k)
            want = np.sort(row)[::-1][:k]
            assert 0 <= passes <= 3
            # all above the threshold, and the first `equal` of those that are it
            assert (row > key).sum() + equal == k and equal <= (row == key).sum() and key <= want[-1]
            assert np.array_equal(np.sort(np.concatenate([row[row > key], row[row == key][:equal]]))[::-1], want)


@pytest.mark.parametrize("kind", ["any", "near", "few", "mostly"])
def test_a_row_that_changes_ends_the_search_too(lib, kind):
    rng, pick = np.random.default_rng(2), random.Random(2)
    for _ in range(400):
        n = pick.choice([2, 50, 4000])
        rows = np.stack([draw(pick.choice([kind, "any", "near", "few"]), n, rng) for _ in range(4)])
        passes, _, equal = search(lib, rows, int(rng.integers(1, n)))
        assert 0 <= passes <= 3 and equal < n


def test_numbers_that_vanish(lib):
    """Every number leaves the range between two passes."""
    rows = np.array([[1, 1 << 31, 0xFFFFFFFF, 5], [7] * 4, [9] * 4])
    rows[1:] = 1 << 20
    for k in (1, 2, 3):
        assert 0 <= search(lib, rows, k)[0] <= 3
    # ... before the first
    out = (ctypes.c_uint32 * 2)()
    row = np.full(4, 3, dtype=np.uint32)
    assert lib.search(ctypes.c_void_p(row.ctypes.data), 1, 4, 2, 100, 200, out) == 1
