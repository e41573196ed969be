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


class Tensor:
    """As much of a device tensor as the calls look at."""

    is_cuda = True

    def __init__(self, dtype, count, device=-1, contiguous=True):
        self.dtype, self.count, self.contiguous = f"torch.{dtype}", count, contiguous
        self.device = type("Device", (), dict(index=device))

    def numel(self):
        return self.count

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 4096


def test_tensors_of_attention_that_do_not_fit_are_refused():
    p, (a, b, c) = host_pool()
    two = p.open(p.register(**dict(ROW, n_q_heads=6)), 8)
    for r, heads in ((a, 4), (two, 6)):
        args = dict(q=Tensor("bfloat16", 1), out=Tensor("bfloat16", 1), lse=Tensor("float32", 1))
        calls = (lambda **k: p.extend([r], [3], **{**args, **k}),
                 lambda **k: p.extend_step([r], [3], Tensor("bfloat16", 1), **{**args, **k}))
        good = dict(slopes=Tensor("float32", heads), doc_begin=Tensor("int32", 3))
        for call in calls:
            with pytest.raises(cpl.CrossPoolError) as e:  # all of it right, but no GPU
                call(**good)
            assert e.value.status == cpl.CP_ESTATE
            for bad in (dict(slopes=Tensor("float32", heads - 1)), dict(slopes=Tensor("float64", heads)),
                        dict(slopes=Tensor("float32", heads, contiguous=False)), dict(doc_begin=Tensor("int32", 2)),
                        dict(doc_begin=Tensor("int64", 3)), dict(doc_begin=Tensor("int32", 3, contiguous=False)),
                        dict(q=Tensor("bfloat16", 1, device=1)), dict(out=Tensor("bfloat16", 1, device=0)),
                        dict(lse=Tensor("float32", 1, device=1)), dict(slopes=Tensor("float32", heads, device=1)),
                        dict(doc_begin=Tensor("int32", 3, device=2)), dict(q=Tensor("bfloat16", 1, contiguous=False))):
                with pytest.raises(ValueError):
                    call(**{**good, **bad})
    for r in (a, b, c, two):
        p.close(r)
    p.destroy()


def test_positions_that_do_not_fit_are_refused():
    rope = cpl.Rope(8, device=-1)
    parts = (cpl.cp_rope_tensor * 1)(cpl.cp_rope_tensor(4096, 4096, 8, 8, 8, 8, 1, 8, 0, cpl.CP_ROPE_BF16))
    parts.tokens, parts.device = 3, 0
    with pytest.raises(cpl.CrossPoolError):
        cpl.cp_rope_apply(rope.handle, parts, Tensor("int32", 3, device=0), stream=0)
    for bad in (Tensor("int32", 3, device=1), Tensor("int32", 4, device=0), Tensor("int64", 3, device=0),
                Tensor("int32", 3, device=0, contiguous=False)):
        with pytest.raises(ValueError):
            cpl.cp_rope_apply(rope.handle, parts, bad, stream=0)
    rope.destroy()


def test_a_destroyed_rotation_is_not_no_rotation():
    """(its handle, None, would store the rows as they are)"""
    p, (a, b, c) = host_pool()
    rope = cpl.Rope(8, device=-1)
    rope.destroy()
    rope.destroy()
    for call in (lambda: p.extend_step([a], [3], 4096, 4096, 4096, 4096, 0, rope=rope),
                 lambda: p.append_rope([a], [3], None, rope, 0), lambda: rope.angles(),
                 lambda: rope.apply(cpl.rope_parts([]), stream=0)):
        with pytest.raises(ValueError):
            call()
    for r in (a, b, c):
        p.close(r)
    p.destroy()


def test_tensors_of_a_rotation_that_meet_are_refused():
    rope = cpl.Rope(8, device=-1)

    def status(*pairs, tokens=2):
        parts = (cpl.cp_rope_tensor * len(pairs))(
            *[cpl.cp_rope_tensor(s, d, 32, 8, 32, 8, 4, 8, 0, cpl.CP_ROPE_BF16) for s, d in pairs])
        parts.tokens = tokens
        with pytest.raises(cpl.CrossPoolError) as e:
            cpl.cp_rope_apply(rope.handle, parts, stream=0)
        return e.value.status

    a, b, c, d = (1 << 20, 2 << 20, 3 << 20, 4 << 20)
    for pairs in (((a, b), (c, b)), ((a, b), (b, c)), ((b, c), (a, b)), ((a, a), (a, b)), ((a, b), (a, a)),
                  ((a, a), (a, a)), ((a, b), (c, d), (b, c))):
        assert status(*pairs) == cpl.CP_EINVAL, pairs
    # sources may be shared, and no tokens meet nowhere (a host-only rotation refuses all, last)
    for pairs in (((a, b), (a, c)), ((a, a), (b, b)), ((a, b), (c, d))):
        assert status(*pairs) == cpl.CP_ESTATE, pairs
    assert status((a, a), (a, a), tokens=0) == cpl.CP_ESTATE
    rope.destroy()
