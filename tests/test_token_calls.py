"""Trees, weights, kept tokens and evictions on the CPU: what a host-only pool counts,
what each call refuses, and launches that fail (a stand-in for the HIP runtime)."""
import ctypes
import os
import random
import subprocess
import sys

import pytest

from paper_2606_24506_amd import crosspool as cpl
from test_failed_launches import SETUP, fake  # noqa: F401  (the stand-in)
from test_fork_truncate import P, ROW, grow, pool

HERE = os.path.dirname(os.path.abspath(__file__))


# ------------------------------------------------ a host-only pool's books


def test_kept_tokens_give_pages_back():
    p = pool()
    m = p.register(**ROW, n_layers=2)
    a = p.open(m, 100)
    grow(p, a, 23)
    before = p.pages(a, layers=2)
    p.keep([a], [17], [2], [0, 3])  # 19 tokens: five pages of six
    assert (p.ctx_len(a), p.position(a)) == (19, 19)
    assert p.pages(a, layers=2).tolist() == before[:, :5].tolist()
    s = p.stats()
    assert (s["pages_used"], s["pages_reserved"]) == (10, 50)
    p.keep([a], [19], [0], [])  # all there is
    p.keep([a], [3], [16], range(16))
    assert (p.ctx_len(a), p.stats()) == (19, s)
    p.keep([a], [0], [0], [])
    assert (p.ctx_len(a), p.position(a), p.stats()["pages_used"]) == (0, 0, 0)
    grow(p, a, 100)
    p.close(a)
    p.destroy()


def test_shared_pages_are_replaced_only_where_rows_move():
    p = pool()
    m = p.register(**ROW)
    a, b = p.open(m, 100), p.open(m, 100)
    grow(p, a, 32)
    p.fork([a], [b])
    was = list(p.pages(a))
    p.keep([b], [10], [9], [0, 1, 2, 3, 4, 10, 11, 12, 13])  # rows from 15 on: pages 3 and 4
    now = list(p.pages(b))
    assert list(p.pages(a)) == was and p.ctx_len(b) == 19
    assert now[:3] == was[:3] and not set(now[3:]) & set(was) and len(now) == 5
    assert p.stats()["pages_used"] == 10
    p.keep([a], [0], [32], range(32))  # nothing goes, nothing moves
    assert list(p.pages(a)) == was
    p.keep([a], [0], [12], range(12))  # whole pages stay shared
    assert list(p.pages(a)) == was[:3]
    for r in (a, b):
        p.close(r)
    assert p.stats()["pages_used"] == p.stats()["pages_reserved"] == 0
    p.destroy()


def test_one_call_for_two_that_share():
    p = pool()
    m = p.register(**ROW)
    a, b = p.open(m, 40), p.open(m, 40)
    grow(p, a, 24)
    p.fork([a], [b])
    was = list(p.pages(a))
    p.keep([a, b], [4, 4], [10, 11], [*range(5, 15), *range(9, 20)])
    pa, pb = list(p.pages(a)), list(p.pages(b))
    assert pa[0] == pb[0] == was[0]
    assert not set(pa[1:]) & set(pb[1:]) and not (set(pa[1:]) | set(pb[1:])) & set(was)
    assert p.stats()["pages_used"] == 1 + 3 + 3
    for r in (a, b):
        p.close(r)
    p.destroy()


def test_budget_and_reservations():
    p = pool(chunks=2, pages_per_chunk=8)  # 16 pages
    m = p.register(**ROW)
    a, b = p.open(m, 8 * P), p.open(m, 8 * P)
    grow(p, a, 8 * P)
    p.fork([a], [b])
    c = p.open(m, 8 * P)  # b's eight pages are a's
    before = p.stats(), list(p.pages(b))
    for keep in ([0, 5, 6, 7], [3], []):
        with pytest.raises(cpl.CrossPoolError) as e:
            p.keep([b], [0], [len(keep)], keep)
        assert e.value.status == cpl.CP_ENOSPC
        assert (p.stats(), list(p.pages(b)), p.ctx_len(b)) == (*before, 8 * P)
    p.close(c)
    p.keep([b], [0], [4], [0, 5, 6, 7])
    grow(p, b, 8 * P - 4)
    assert p.stats()["pages_used"] == p.stats()["pages_reserved"] == 16
    for r in (a, b):
        p.close(r)
    p.destroy()


@pytest.mark.parametrize("backing", [0, 1])
@pytest.mark.parametrize("seed", range(6))
def test_random_calls_against_a_page_count(seed, backing):
    """Forks, appends, cuts and kept tokens: pages in use are those that some request shows,
    each page inside its request's length, and no page of two kept paths is the same."""
    rng = random.Random(seed)
    kw = dict(backing=cpl.CP_BACKING_VIRTUAL) if backing else {}
    try:
        p = pool(chunks=40, pages_per_chunk=8, **kw)
    except cpl.CrossPoolError as e:
        pytest.skip(str(e))
    layers = rng.choice([1, 3])
    m = p.register(**ROW, n_layers=layers)
    ids, lens = [], {}
    for _ in range(300):
        op = rng.random()
        if len(ids) < 5 and op < 0.2:
            try:
                ids.append(p.open(m, 40))
                lens[ids[-1]] = 0
            except cpl.CrossPoolError:
                pass
        elif not ids:
            continue
        elif op < 0.4:
            r = rng.choice(ids)
            n = rng.randint(0, 40 - lens[r])
            grow(p, r, n)
            lens[r] += n
        elif op < 0.55 and len(ids) > 1:
            a, b = rng.sample(ids, 2)
            try:
                p.truncate([b], [0])
                lens[b] = 0
                p.fork([a], [b])
                lens[b] = lens[a]
            except cpl.CrossPoolError as e:
                assert e.status == cpl.CP_ENOSPC
        elif op < 0.9:
            some = rng.sample(ids, rng.randint(1, len(ids)))
            first = [rng.randint(0, lens[r]) for r in some]
            lists = [sorted(rng.sample(range(lens[r] - f), rng.randint(0, lens[r] - f))) for r, f in zip(some, first)]
            before = [p.pages(r, layers=layers).tolist() for r in ids]
            try:
                p.keep(some, first, [len(x) for x in lists], [t for x in lists for t in x])
                for r, f, x in zip(some, first, lists):
                    lens[r] = f + len(x)
            except cpl.CrossPoolError as e:
                assert e.status == cpl.CP_ENOSPC
                assert before == [p.pages(r, layers=layers).tolist() for r in ids]
        elif len(ids) > 2:
            r = ids.pop(rng.randrange(len(ids)))
            p.close(r)
            del lens[r]
        shown = set()
        for r in ids:
            assert p.ctx_len(r) == lens[r] == p.position(r)
            pages = p.pages(r, layers=layers).reshape(-1).tolist()
            assert len(set(pages)) == len(pages) == layers * ((lens[r] + P - 1) // P)
            shown |= set(pages)
        s = p.stats()
        assert s["pages_used"] == len(shown) <= s["pages_reserved"]
    for r in ids:  # what was admitted can be filled
        p.truncate([r], [0])
        grow(p, r, 40)
    for r in ids:
        p.close(r)
    assert p.stats()["pages_used"] == p.stats()["pages_reserved"] == 0
    p.destroy()


def test_refusals_of_keep():
    p = pool()
    m = p.register(**ROW)
    a, b = p.open(m, 40), p.open(m, 40)
    grow(p, a, 20)
    before = p.stats()
    for ids, first, lists in (([a], [21], [[]]), ([a], [-1], [[]]), ([a], [5], [[15]]), ([a], [5], [[-1]]),
                              ([a], [5], [[3, 3]]), ([a], [5], [[4, 2]]), ([a], [20], [[0]]), ([a, a], [0, 0], [[1], [2]]),
                              ([a, b], [0, 0], [[1], [0]]), ([99], [0], [[]])):
        with pytest.raises(cpl.CrossPoolError) as e:
            p.keep(ids, first, [len(x) for x in lists], [t for x in lists for t in x])
        assert e.value.status == cpl.CP_EINVAL
    for args in (([a], [0], [2], [1]), ([a], [0, 1], [1], [1]), ([a], [0], [], [])):
        with pytest.raises(ValueError):
            p.keep(*args)
    lib, one = cpl.LIB, (ctypes.c_int64 * 1)(0)
    ids, n = (ctypes.c_int32 * 1)(a), (ctypes.c_int32 * 1)(1)
    assert lib.cp_request_keep(p.handle, 1, ids, None, n, n, None) == cpl.CP_EINVAL
    assert lib.cp_request_keep(p.handle, 1, ids, one, None, n, None) == cpl.CP_EINVAL
    assert lib.cp_request_keep(p.handle, 1, ids, one, n, None, None) == cpl.CP_EINVAL
    n[0] = -1
    assert lib.cp_request_keep(p.handle, 1, ids, one, n, None, None) == cpl.CP_EINVAL
    assert lib.cp_request_keep(None, 1, ids, one, n, None, None) == cpl.CP_EINVAL
    assert lib.cp_request_position(p.handle, 99, one) == cpl.CP_EINVAL
    assert lib.cp_request_position(p.handle, a, None) == cpl.CP_EINVAL
    p.keep([], [], [], [])
    assert p.stats() == before and p.ctx_len(a) == 20
    # nothing to choose from or to ask
    assert lib.cp_kv_evict(p.handle, 1, ids, one, None, None, None) == cpl.CP_ESTATE
    assert lib.cp_attn_weights(p.handle, 1, ids, n, None, None, 0, 0.0, None, None, None, None) == cpl.CP_ESTATE
    p.close(a)
    p.close(b)
    p.destroy()


class Rows:
    """As much of a tensor on the GPU as token_rows looks at."""

    def __init__(self, *shape, dtype="float32", device=0, is_cuda=True, stride=None):
        self.shape, self.dtype, self.device, self.is_cuda = shape, f"torch.{dtype}", device, is_cuda
        self.strides = stride or tuple(shape[-1] ** (len(shape) - 1 - i) for i in range(len(shape)))

    def dim(self):
        return len(self.shape)

    def stride(self, i):
        return self.strides[i]

    def data_ptr(self):
        return 1 << 20


@pytest.mark.parametrize("bad", [[Rows(4)], [Rows(1, 2, 3, 4)], [Rows(2, 4, stride=(1, 2))], [Rows(2, 4, dtype="float16")],
                                 [Rows(2, 4), Rows(2, 4, dtype="int32")], [Rows(2, 4, is_cuda=False)],
                                 [Rows(2, 4), Rows(2, 4, device=1)]])
def test_rows_that_are_none(bad):
    with pytest.raises(ValueError):
        cpl.token_rows(bad)


# --------------------------------------- calls on a device that stands still

MORE = SETUP + """
from paper_2606_24506_amd.crosspool import LIB, cp_tree, cp_token_rows, cp_evict_opts, cp_extend_opts
I32, I64 = lambda *x: (ctypes.c_int32 * max(1, len(x)))(*x), lambda *x: (ctypes.c_int64 * max(1, len(x)))(*x)
by = ctypes.byref
LAYERS, HKV = 2, 3
room = (ctypes.c_char * (1 << 20))()
R = (ctypes.addressof(room) + 255) // 256 * 256

def heads_pool(**kw):
    p = cpl.Pool(page_tokens=P, pool_bytes=32 << 20, chunk_bytes=1 << 16, device=0, **kw)
    return p, p.register(cpl.CP_KIND_GQA, 2 * HKV, HKV, head_dim=64, n_layers=LAYERS)

def rec(n, at=0, head=None, layer=None, length=None, data=None):
    head = n if head is None else head
    return cp_token_rows(R + at if data is None else data, n if length is None else length, head, HKV * head if layer is None else layer)

def rows(*x):
    return (cp_token_rows * len(x))(*x)

def refused(rc, word):
    text = LIB.cp_last_error().decode()
    assert rc == cpl.CP_EINVAL and word in text, (rc, text, word)
"""

REFUSALS = {
    "trees": """
p, m = pool()
a, b = p.open(m, 200), p.open(m, 200)
p.append([a, b], [150, 10], at, 0)
before = p.stats()
def tree(words=4, mask=at, depth=at):
    return cp_tree(mask, words, 0, depth)
def call(t, ids=(a, b), n_q=(100, 10), q=at, out=at, lse=at, o=None):
    return LIB.cp_attn_tree(p.handle, len(ids), I32(*ids), I32(*n_q), q, out, lse, by(t) if t else None, None, by(o) if o else None)
def step(t, ids=(a, b), n_new=(20, 10), rows=at, o=None):
    return LIB.cp_attn_tree_step(p.handle, len(ids), I32(*ids), I32(*n_new), rows, at, at, at, by(t) if t else None, None,
                                 by(o) if o else None)
o = cp_extend_opts()
o.prefix = ctypes.cast(I32(0, 0), ctypes.c_void_p).value
for f in (call, step):
    refused(f(None), "tree")
    for w in (0, -1, 129):
        refused(f(tree(w)), "words")
    refused(f(tree(mask=None)), "null")
    refused(f(tree(depth=None)), "null")
    refused(f(tree(mask=at + 2)), "aligned")
    refused(f(tree(depth=at + 1)), "aligned")
    refused(f(tree(), o=o), "prefix")
refused(call(tree(3)), "fit")
refused(step(tree(1), n_new=(33, 10)), "fit")
refused(call(tree(), n_q=(151, 0)), "context")
refused(call(tree(), q=None), "null")
refused(call(tree(), q=at + 8), "align")
refused(step(tree(), n_new=(-1, 0)), "")
assert (p.stats(), p.ctx_len(a), p.ctx_len(b)) == (before, 150, 10)
assert call(tree()) == cpl.CP_OK and call(tree(mask=None, depth=None), n_q=(0, 0)) == cpl.CP_OK
def build(n_tok, parents=at, words=4, mask=R, depth=R + (1 << 18), n=None, device=0):
    return LIB.cp_tree_build(device, len(n_tok) if n is None else n, I32(*n_tok), parents, words, mask, depth, None)
for w in (0, 129):
    refused(build((3,), words=w), "words")
refused(build((129,)), "")
refused(build((-1,)), "")
refused(build((3,), n=-1), "")
for k in ("parents", "mask", "depth"):
    refused(build((3,), **{k: None}), "null")
    refused(build((3,), **{k: R + (1 << 17) + 2}), "aligned")
refused(build((3,), mask=at), "overlap")
refused(build((3,), depth=R + 4), "overlap")
refused(build((3,), device=1), "device")
assert LIB.cp_tree_build(0, 1, None, at, 4, R, R + 4096, None) == cpl.CP_EINVAL
launches = fake.fake_launches()
assert build(()) == build((0, 0), None, 1, None, None) == cpl.CP_OK and fake.fake_launches() == launches
assert build((128, 0, 5)) == cpl.CP_OK
usable(p, [a, b])
""",
    "weights": """
p, m = heads_pool()
a, b = p.open(m, 64), p.open(m, 64)
p.append([a, b], [40, 9], at, 0)
other = p.register(cpl.CP_KIND_GQA, 2, 1, head_dim=64)
c = p.open(other, 8)
before = p.stats()
ok = rows(rec(40), rec(9, 1 << 16))
def call(new=ok, old=None, ids=(a, b), n_q=(3, 1), q=at, lse=at, layer=0, decay=1.0, **kw):
    o = cp_extend_opts()
    for k, v in kw.items():
        setattr(o, k, v)
    return LIB.cp_attn_weights(p.handle, len(ids), I32(*ids) if ids else None, I32(*n_q) if n_q is not None else None, q, lse,
                               layer, decay, old, new, None, by(o))
refused(call(ids=(), n_q=()), "")
refused(call(ids=(a, a)), "")
refused(call(ids=(a, 99)), "")
refused(call(ids=(a, c)), "model")
refused(call(n_q=None), "null")
refused(call(new=None), "null")
refused(call(n_q=(41, 0)), "context")
refused(call(n_q=(-1, 0)), "context")
refused(call(q=None), "null")
refused(call(lse=None), "null")
refused(call(q=at + 8), "aligned")
refused(call(lse=at + 2), "aligned")
for layer in (-1, LAYERS):
    refused(call(layer=layer), "layer")
for decay in (-0.5, 1.5, float("nan"), float("inf")):
    refused(call(decay=decay), "decay")
for k, v in (("softcap", -1.0), ("softcap", float("nan")), ("window", -1), ("num_splits", -1), ("path", 7), ("rope", at),
             ("slopes", at + 1), ("doc_begin", at + 2), ("prefix", ctypes.cast(I32(0, -1), ctypes.c_void_p).value)):
    refused(call(**{k: v}), "")
refused(call(rows(rec(40, data=0), rec(9, 1 << 16))), "null")
refused(call(rows(rec(40, 2), rec(9, 1 << 16))), "aligned")
refused(call(rows(rec(39), rec(9, 1 << 16))), "needed")
refused(call(rows(rec(40, head=39), rec(9, 1 << 16))), "heads overlap")
refused(call(rows(rec(40, head=-40), rec(9, 1 << 16))), "heads overlap")
refused(call(rows(rec(40, layer=3 * 40 - 1), rec(9, 1 << 16))), "layers overlap")
refused(call(rows(rec(40), rec(9, 4 * 3 * 40 - 4))), "overlap")  # the last of the first's row
refused(call(ok, rows(rec(40, 4), rec(9, 1 << 16))), "overlap")  # not quite the same
refused(call(ok, rows(rec(9, 1 << 16), rec(40))), "")            # another entry's
assert (p.stats(), p.ctx_len(a)) == (before, 40)
# slices that lie between one another's rows, other layers' places, the same, and what is not read
assert call(ok, ok) == cpl.CP_OK
assert call(rows(rec(40, head=64, layer=512), rec(9, 4 * 40, head=64, layer=512))) == cpl.CP_OK
refused(call(rows(rec(40, head=64, layer=512), rec(9, 4 * 39, head=64, layer=512))), "overlap")
assert call(ok, rows(rec(40, 4 * 3 * 40), rec(9, 1 << 17))) == cpl.CP_OK  # layer 1 of one is beside layer 0 of the other
assert call(ok, rows(rec(1, 2), rec(1, 2)), decay=0.0) == cpl.CP_OK
assert call(n_q=(0, 0), q=None, lse=None) == cpl.CP_OK
p.append([c], [1], at, 0)
p.close(c)
usable(p, [a, b])
""",
    "evict": """
p, m = heads_pool()
a, b = p.open(m, 64), p.open(m, 64)
p.append([a, b], [40, 9], at, 0)
other = p.register(cpl.CP_KIND_GQA, 2, 1, head_dim=64)
c = p.open(other, 8)
before = p.stats()
W = rows(rec(40), rec(9, 1 << 16))
def call(w=W, n_keep=(20, 9), ids=(a, b), first=0, last=0, new=None, kept=None):
    ad = lambda x: None if x is None else ctypes.addressof(x)
    o = cp_evict_opts(first, last, ad(new), ad(kept))
    return LIB.cp_kv_evict(p.handle, len(ids), I32(*ids), I64(*n_keep) if n_keep else None, w, by(o), None)
refused(call(n_keep=None), "null")
refused(call(None), "null")
refused(call(ids=(a, a)), "")
refused(call(ids=(a, c)), "model")
refused(call(n_keep=(-1, 0)), "n_keep")
refused(call(first=-1), "first")
refused(call(last=-1), "last")
refused(call(first=11, last=10), "more than")
refused(call(first=2**31 - 1, last=2**31 - 1), "more than")
refused(call(rows(rec(40, data=0), rec(9, 1 << 16))), "null")
refused(call(rows(rec(40, length=39), rec(9, 1 << 16))), "needed")
refused(call(rows(rec(40, head=30), rec(9, 1 << 16))), "heads overlap")
refused(call(rows(rec(40, layer=100), rec(9, 1 << 16))), "layers overlap")
refused(call(new=rows(rec(20), rec(9, 1 << 16))), "needed")  # (its rest becomes 0)
refused(call(new=rows(rec(40, 4), rec(9, 1 << 16))), "overlap")
refused(call(kept=W), "overlap")
refused(call(new=W, kept=rows(rec(20), rec(9, 1 << 17))), "overlap")
refused(call(kept=rows(rec(19, 1 << 17), rec(9, 1 << 18))), "needed")
assert (p.stats(), p.ctx_len(a), p.position(a)) == (before, 40, 40)
launches = fake.fake_launches()
assert LIB.cp_kv_evict(p.handle, 0, None, None, None, None, None) == cpl.CP_OK and fake.fake_launches() == launches
fake.fake_no_memory(1)
assert call() == cpl.CP_ENOMEM
fake.fake_no_memory(0)
assert (p.stats(), p.ctx_len(a)) == (before, 40)
assert call(first=10, last=10, new=W, kept=rows(rec(20, 1 << 17), rec(9, 1 << 18))) == cpl.CP_OK
assert (p.ctx_len(a), p.position(a), p.ctx_len(b), p.position(b)) == (20, 40, 9, 9)
d = p.open(m, 64)
p.fork([a], [d], [12], 0)
assert (p.ctx_len(d), p.position(d)) == (12, 32)
p.append([d], [1], at, 0)
p.truncate([d], [5], 0)
assert p.position(d) == 25
assert call(ids=(d,), n_keep=(0,), w=rows(rec(5))) == cpl.CP_OK
assert (p.ctx_len(d), p.position(d)) == (0, 25)
p.truncate([a], [0], 0)
assert p.position(a) == 0
p.append([a], [20], at, 0)
p.close(d)
p.close(c)
usable(p, [a, b])
""",
    "tokens in flight": """
p, m = heads_pool()
a, b = p.open(m, 64), p.open(m, 64)
p.append([a, b], [40, 9], at, 0)
p.extend_step([a], [2], at, at, at, at, 0)  # of two layers
W = rows(rec(42), rec(9, 1 << 16))
assert status(p.keep, [a], [0], [1], [0], 0)[0] == cpl.CP_EINVAL
refused(LIB.cp_kv_evict(p.handle, 1, I32(a), I64(5), W, None, None), "flight")
def weights(layer, n_q):
    return LIB.cp_attn_weights(p.handle, 1, I32(a), I32(n_q), at, at, layer, 1.0, None, W, None, None)
assert weights(0, 42) == weights(1, 40) == cpl.CP_OK  # layer 0 has them
refused(weights(1, 41), "context")
p.extend_step([a], [2], at, at, at, at, 0)
assert weights(1, 42) == cpl.CP_OK
usable(p, [a, b])
""",
}


@pytest.mark.parametrize("case", sorted(REFUSALS))
def test_refusals(case, fake):  # noqa: F811
    run(MORE + REFUSALS[case], fake)


FAILURES = {
    "tree step, the append": """
p, m = pool()
a = p.open(m, 40)
p.append([a], [10], at, 0)
t = cp_tree(at, 1, 0, at)
fake.fake_fail_in(1)
assert LIB.cp_attn_tree_step(p.handle, 1, I32(a), I32(3), at, at, at, at, by(t), None, None) == cpl.CP_EHIP
unusable(p, [a], m)
""",
    "tree step, the attention": """
p, m = pool()
a = p.open(m, 40)
p.append([a], [10], at, 0)
t = cp_tree(at, 1, 0, at)
fake.fake_fail_in(2)
assert LIB.cp_attn_tree_step(p.handle, 1, I32(a), I32(3), at, at, at, at, by(t), None, None) == cpl.CP_EHIP
unusable(p, [a], m)
""",
    "trees and weights change nothing": """
p, m = heads_pool()
a = p.open(m, 40)
p.append([a], [10], at, 0)
t = cp_tree(at, 1, 0, at)
fake.fake_fail_in(1)
assert LIB.cp_attn_tree(p.handle, 1, I32(a), I32(3), at, at, at, by(t), None, None) == cpl.CP_EHIP
fake.fake_fail_in(1)
assert LIB.cp_tree_build(0, 1, I32(3), at, 1, R, R + 4096, None) == cpl.CP_EHIP
for n_q in (1, 10):
    fake.fake_fail_in(1)
    assert LIB.cp_attn_weights(p.handle, 1, I32(a), I32(n_q), at, at, 0, 1.0, None, rows(rec(10)), None, None) == cpl.CP_EHIP
usable(p, [a])
""",
    "keep, the moves": """
p, m = pool(layers=3)
a = p.open(m, 40)
p.append([a], [20], at, 0)
fake.fake_fail_in(1)
assert status(p.keep, [a], [3], [3], [2, 9, 11], 0)[0] == cpl.CP_EHIP
unusable(p, [a], m)
""",
    "keep, the replaced pages": """
p, m = pool(layers=3)
a, b = p.open(m, 40), p.open(m, 40)
p.append([a], [20], at, 0)
p.fork([a], [b], None, 0)
fake.fake_fail_in(1)
assert status(p.keep, [b], [3], [3], [2, 9, 11], 0)[0] == cpl.CP_EHIP
unusable(p, [a, b], m)
""",
    "evict, the choice": """
p, m = heads_pool()
a = p.open(m, 40)
p.append([a], [20], at, 0)
fake.fake_fail_in(1)
assert LIB.cp_kv_evict(p.handle, 1, I32(a), I64(7), rows(rec(20)), None, None) == cpl.CP_EHIP
unusable(p, [a], m)
""",
    "evict, the moves": """
p, m = heads_pool()
a, b = p.open(m, 40), p.open(m, 40)
p.append([a], [20], at, 0)
p.fork([a], [b], None, 0)
fake.fake_fail_in(2)
assert LIB.cp_kv_evict(p.handle, 1, I32(b), I64(7), rows(rec(20)), None, None) == cpl.CP_EHIP
unusable(p, [a, b], m)
""",
    "an error left behind by another call": """
p, m = heads_pool()
a = p.open(m, 40)
p.append([a], [20], at, 0)
before = p.stats()
for fn in (lambda: status(p.keep, [a], [3], [3], [2, 9, 11], 0)[0],
           lambda: LIB.cp_kv_evict(p.handle, 1, I32(a), I64(7), rows(rec(20)), None, None)):
    fake.fake_leave_error(1)  # an invalid value
    assert fn() == cpl.CP_EHIP
    assert (p.stats(), p.ctx_len(a), p.position(a)) == (before, 20, 20)
usable(p, [a])
""",
    "an unusable pool": """
p, m = heads_pool()
a = p.open(m, 40)
p.append([a], [20], at, 0)
fake.fake_fail_in(1)
assert status(p.keep, [a], [3], [3], [2, 9, 11], 0)[0] == cpl.CP_EHIP
t = cp_tree(at, 1, 0, at)
assert status(p.keep, [a], [0], [1], [0], 0)[0] == cpl.CP_ESTATE
for rc in (LIB.cp_kv_evict(p.handle, 1, I32(a), I64(2), rows(rec(20)), None, None),
           LIB.cp_attn_weights(p.handle, 1, I32(a), I32(1), at, at, 0, 1.0, None, rows(rec(20)), None, None),
           LIB.cp_attn_tree(p.handle, 1, I32(a), I32(1), at, at, at, by(t), None, None),
           LIB.cp_attn_tree_step(p.handle, 1, I32(a), I32(1), at, at, at, at, by(t), None, None)):
    assert rc == cpl.CP_ESTATE
unusable(p, [a], m)
""",
}


@pytest.mark.parametrize("case", sorted(FAILURES))
def test_failed_launches(case, fake):  # noqa: F811
    run(MORE + FAILURES[case], fake)


def run(program, stand_in):
    res = subprocess.run([sys.executable, "-c", program, stand_in], cwd=os.path.dirname(HERE), capture_output=True, text=True,
                         timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
