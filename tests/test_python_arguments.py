"""What the Python calls take as host arrays and refuse as device tensors (no GPU)."""
import ctypes

import numpy as np
import pytest

from paper_2606_24506_amd import crosspool as cpl

ROW = dict(kind=cpl.CP_KIND_GQA, n_q_heads=4, n_kv_heads=1, head_dim=64)


def host_pool(n=3):
    p = cpl.Pool(page_tokens=4, pool_bytes=1 << 20, chunk_bytes=1 << 13, device=-1)
    m = p.register(**ROW)
    return p, [p.open(m, 40) for _ in range(n)]


@pytest.mark.parametrize("make", [cpl.i32_array, cpl.i64_array, list, tuple, np.array, lambda x: np.array(x, np.int32),
                                  lambda x: np.array([x, x], np.int32).T[:, 0], lambda x: (ctypes.c_uint8 * len(x))(*x)])
def test_integers_of_any_array_type(make):
    p, (a, b, c) = host_pool()
    p.append(make([a, b]), make([21, 17]), None)
    p.fork(make([a, a][:1]), make([c]), make([9]))
    assert [p.ctx_len(r) for r in (a, b, c)] == [21, 17, 9]
    p.truncate(make([a, b, c]), make([10, 0, 6]))
    assert [p.ctx_len(r) for r in (a, b, c)] == [10, 0, 6]
    for r in (a, b, c):
        p.close(r)
    p.destroy()


def test_integers_out_of_range_are_refused():
    p, (a, b, c) = host_pool()
    for bad in (cpl.i64_array([1 << 32]), [1 << 32], np.array([-(1 << 31) - 1])):
        with pytest.raises((ValueError, OverflowError)):
            p.append([a], bad, None)
        with pytest.raises((ValueError, OverflowError)):
            p.append(bad, [1], None)
    with pytest.raises((ValueError, OverflowError)):
        p.truncate([a], [1 << 64])
    assert p.ctx_len(a) == 0
    for r in (a, b, c):
        p.close(r)
    p.destroy()
