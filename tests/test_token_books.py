"""Requests cut to some of their tokens, on the CPU: what a call does that its
neighbours in the call, earlier work of the stream or its size could change (a
stand-in for the HIP runtime, tests/c/queued_hip.cpp, or a host-only pool)."""
import os
import random
import shutil
import subprocess

import pytest

from paper_2606_24506_amd import build
from paper_2606_24506_amd import crosspool as cpl
from test_fork_truncate import P, ROW, grow, pool
from test_token_calls import MORE, run

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def queued(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    out = str(tmp_path_factory.mktemp("queued") / "queued_hip.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", build.CSRC,
                    os.path.join(HERE, "c", "queued_hip.cpp"), "-o", out], check=True)
    return out


def test_every_kept_row_of_a_call_of_many_workgroups_moves(queued):
    """Three requests of 1,024 layers and the widest rows are more workgroups than a launch
    takes, and the third's list does not fit the second launch's arguments whole."""
    run(MORE + """
P = 128
p = cpl.Pool(page_tokens=P, pool_bytes=3200 << 26, chunk_bytes=1 << 26, device=0, device_mem=at, max_requests=4)
m = p.register(cpl.CP_KIND_GQA, 256, 256, head_dim=512, n_layers=1024)
ids = [p.open(m, P) for _ in range(3)]
p.append(ids, [P] * 3, at, 0)
seen, launches = [], []
buf = ((ctypes.c_int64 * 3) * 1024)()
@ctypes.CFUNCTYPE(None, ctypes.c_void_p)
def launched(args):
    n = fake.kept_rows(ctypes.c_void_p(args), buf, 1024)
    launches.append(n)
    seen.extend(tuple(x) for x in buf[:n])
fake.watch_launches(launched)
keep = list(range(P - 100, P))
p.keep(ids, [0] * 3, [100] * 3, keep * 3, 0)
fake.watch_launches(None)
bases = sorted({x[0] for x in seen})
assert len(bases) == 3 and len(launches) > 1
assert sorted(seen) == sorted((b, k, t) for b in bases for k, t in enumerate(keep)), launches
for r in ids:
    p.close(r)
p.destroy()
""", queued)


EMPTIED = """
p, m = heads_pool()
a, b, c = p.open(m, 64), p.open(m, 64), p.open(m, 64)
W = lambda n: rows(rec(n))
def emptied(r, n):  # of n tokens by an eviction
    p.append([r], [n], at, 0)
    assert LIB.cp_kv_evict(p.handle, 1, I32(r), I64(0), W(n), None, None) == cpl.CP_OK
    assert (p.ctx_len(r), p.position(r)) == (0, n)
"""


@pytest.mark.parametrize("cut, of_b, of_c", [
    ("p.truncate([a], [0], 0)", 10, 5), ("p.keep([a], [0], [0], [], 0)", 10, 5),
    ("p.truncate([b, a], [9, 0], 0)", 9, 5), ("p.keep([b, a], [9, 0], [0, 0], [], 0)", 9, 5),
    ("p.truncate([b, a], [10, 0], 0)", 10, 5), ("p.keep([b, a], [0, 0], [10, 0], range(10), 0)", 10, 5),
    ("p.truncate([a, c], [0, 0], 0)", 10, 0), ("p.keep([c, a], [0, 0], [0, 0], [], 0)", 10, 0)])
def test_a_request_cut_to_nothing_starts_at_0(cut, of_b, of_c, queued):
    """... also one that an eviction had left nothing of, alone and in company: new keys are
    turned by their places from 0 on."""
    run(MORE + EMPTIED + f"""
p.append([b], [10], at, 0)
emptied(a, 20)
emptied(c, 5)
{cut}
assert (p.ctx_len(a), p.position(a)) == (0, 0)
assert (p.position(b), p.ctx_len(b), p.position(c), p.ctx_len(c)) == ({of_b}, {of_b}, {of_c}, 0)
p.append([a], [7], at, 0)
assert p.position(a) == 7
usable(p, [b, a, c])
""", queued)


def test_an_evicted_request_keeps_its_position_otherwise(queued):
    run(MORE + EMPTIED + """
emptied(a, 20)
p.truncate([b], [0], 0)
p.keep([], [], [], [], 0)
p.truncate([], [], 0)
assert (p.ctx_len(a), p.position(a)) == (0, 20)
p.append([a], [7], at, 0)
assert p.position(a) == 27
p.truncate([a], [3], 0)
assert p.position(a) == 23
p.keep([a], [0], [2], [0, 2], 0)
assert p.position(a) == 22
p.append([b], [10], at, 0)
usable(p, [b, a, c])
""", queued)


STAGED = """
p = cpl.Pool(page_tokens=P, pool_bytes=64 << 20, chunk_bytes=1 << 16, device=0)
m = p.register(cpl.CP_KIND_GQA, 2 * HKV, HKV, head_dim=64, n_layers=LAYERS)
def evict(r, n, keep):
    w = (ctypes.c_float * (n * HKV * LAYERS))()
    x = rows(cp_token_rows(ctypes.addressof(w), n, n, n * HKV))
    assert LIB.cp_kv_evict(p.handle, 1, I32(r), I64(keep), x, None, None) == cpl.CP_OK
fake.late_copies(1)
"""
CLOSE = """
for r in ids:
    p.close(r)
p.destroy()
"""
REWRITES = {
    "a prompt that a fork keeps is evicted, its entries being on the way": """
ids = a, b = [p.open(m, 4000) for _ in range(2)]
p.append([a], [4000], at, 0)
p.fork([a], [b], None, 0)
evict(a, 4000, 1600)
""",
    "branches evicted twice": """
ids = a, b, c = [p.open(m, 4000) for _ in range(3)]
fake.late_copies(0)
p.append([a], [4000], at, 0)
fake.late_copies(1)
p.fork([a], [b], None, 0)
evict(b, 4000, 2400)
p.fork([b], [c], None, 0)
evict(b, 2400, 2000)
""",
    "drafted rows on the way are dropped, and placed on other pages": """
ids = a, b = [p.open(m, 400) for _ in range(2)]
fake.late_copies(0)
p.append([a, b], [4, 4], at, 0)
fake.late_copies(1)
for _ in range(LAYERS):
    p.extend_step([a, b], [9, 9], at, at, at, at, 0)
p.truncate([a, b], [4, 4], 0)
for _ in range(LAYERS):
    p.extend_step([b, a], [9, 9], at, at, at, at, 0)
""",
    "an append on the way is dropped, and its pages are another's then": """
ids = a, b = [p.open(m, 2000) for _ in range(2)]
p.append([a], [2000], at, 0)
p.truncate([a], [0], 0)
p.append([b], [2000], at, 0)
p.append([a], [2000], at, 0)
""",
}


@pytest.mark.parametrize("case", sorted(REWRITES))
def test_page_table_entries_on_the_way_do_not_change(case, queued):
    """New entries go to the device by copies that run behind the stream's earlier work, from
    memory that the host fills again for later calls."""
    run(MORE + STAGED + REWRITES[case] + """
fake.hipDeviceSynchronize()
assert fake.copies() > 1
assert fake.changed_copies() == 0, fake.changed_copies()
""" + CLOSE, queued)


BIG = STAGED.replace("64 << 20", "2 << 30") + """
ids = [p.open(m, 4000) for _ in range(40)]
waited = fake.host_waits()
"""


def test_copies_on_the_way_wait_for_memory_alone(queued):
    run(MORE + BIG + """
def fill(n):
    for r in ids:
        p.append([r], [n], at, 0)
fill(1600)
assert (fake.copies(), fake.host_waits()) == (40, waited)
for i in range(1, 12):  # 56,000 entries each time, of 262,144 that there is memory for
    p.truncate(ids, [0] * 40, 0)
    fill(1600)
assert fake.copies() == 480 and waited + 2 <= fake.host_waits() <= waited + 3
for order in (ids, ids[::-1], ids):  # one copy over every plane: memory grows once
    waited = fake.host_waits()
    p.truncate(ids, [1600] * 40, 0)
    p.append(order, [2400] * 40, at, 0)
    assert fake.host_waits() == waited
fake.hipDeviceSynchronize()
assert (fake.copies(), fake.changed_copies()) == (483, 0)
""" + CLOSE, queued)


def test_without_memory_a_copy_has_run_when_the_call_returns(queued):
    run(MORE + BIG + """
ids += [p.open(m, 4000) for _ in range(120)]  # 320,000 entries
fake.fake_no_memory(1)
p.append(ids, [4000] * 160, at, 0)
assert (fake.copies(), fake.host_waits()) == (1, waited + 1)
p.truncate(ids, [0] * 160, 0)
p.append(ids[::-1], [4000] * 160, at, 0)
assert (fake.copies(), fake.host_waits(), fake.changed_copies()) == (2, waited + 2, 0)
fake.fake_no_memory(0)
""" + CLOSE, queued)


def test_copies_into_graphs_read_the_table(queued):
    """... as it was last copied, at every replay, and wait for nothing."""
    run(MORE + STAGED + """
ids = a, b = [p.open(m, 2000) for _ in range(2)]
fake.capturing(1)
waited = fake.host_waits()
p.append([a], [2000], at, 0)
fake.capturing(0)
p.truncate([a], [0], 0)
p.append([b], [2000], at, 0)
p.append([a], [2000], at, 0)
assert fake.host_waits() == waited
fake.hipDeviceSynchronize()
assert fake.changed_copies() == 1  # the graph's finds what is there now
""" + CLOSE, queued)


# ------------------------------------------------------- budgets of a call


def test_a_prompt_and_its_fork_are_cut_in_one_call():
    """Pages that only the call's requests show go back to the pool, and owe nothing."""
    p = pool(chunks=2, pages_per_chunk=8)  # 16 pages
    m = p.register(**ROW)
    a, b = p.open(m, 8 * P), p.open(m, 8 * P)
    for cut in ("keep", "truncate"):
        grow(p, a, 8 * P)
        p.fork([a], [b])
        if cut == "keep":
            p.keep([a, b], [0, 0], [P, P], [*range(P)] * 2)
        else:
            p.truncate([a, b], [P, P])
        assert p.pages(a).tolist() == p.pages(b).tolist()
        assert (p.stats()["pages_used"], p.stats()["pages_reserved"]) == (1, 15)
        p.truncate([a, b], [0, 0])
    grow(p, a, 8 * P)
    p.fork([a], [b])
    p.keep([a, b], [0, 0], [2, 3], [0, 9, 1, 2, 31])  # a page of its own each, beside the eight
    assert not set(p.pages(a)) & set(p.pages(b)) and p.stats()["pages_reserved"] == 16
    for r in (a, b):
        grow(p, r, 8 * P - p.ctx_len(r))
        p.close(r)
    p.destroy()


def test_an_empty_stack_has_nothing_to_give_back():
    """Replacements beyond what open requests may still take ask no device for pages."""
    p = pool(chunks=2, pages_per_chunk=8, device_pages=1)
    m = p.register(**ROW)
    a, b = p.open(m, 3 * P), p.open(m, 3 * P)
    grow(p, a, 3 * P)
    p.fork([a], [b])
    p.keep([a, b], [0, 0], [11, 11], [*range(1, 12)] * 2)
    assert not set(p.pages(a)) & set(p.pages(b)) and p.stats()["pages_used"] == p.stats()["pages_reserved"] == 6
    for r in (a, b):
        p.close(r)
    p.destroy()


def cut_books(pages, reserve, first, lists):
    """(pages promised after a call, pages that stand beside one another in it) from the pages
    of every request, for the requests that the call cuts."""
    users = {}
    for x in pages.values():
        for page in x:
            users[page] = users.get(page, 0) + 1
    had, own, shown = dict(users), 0, sum(len(x) for x in pages.values())
    for r, f, keep in zip(lists, first, lists.values()):
        stay = sum(t == k for k, t in enumerate(keep))
        last = -(-(f + len(keep)) // P)
        k0 = min((f + stay) // P, last)
        moved = [page for page in pages[r][k0:last] if had[page] > 1]
        own += len(moved)
        shown -= len(pages[r]) - last
        for page in moved + pages[r][last:]:
            users[page] -= 1
    return sum(n > 0 for n in users.values()) + own + reserve * len(pages) - shown, len(users) + own


def test_only_calls_that_the_budget_cannot_hold_are_refused():
    refused, together = (sum(x) for x in zip(*map(random_cuts, range(12))))
    assert refused > 20 and together > 100


def random_cuts(seed):
    """(calls refused, calls that cut several requests that share)"""
    rng = random.Random(seed)
    total, reserve = 24, 10
    p = pool(chunks=total // 8, pages_per_chunk=8)
    m = p.register(**ROW)
    ids, refused, together = [], 0, 0
    for _ in range(400):
        op = rng.random()
        if op < 0.3 and len(ids) < 6:
            try:
                ids.append(p.open(m, reserve * P))
                if len(ids) > 1:
                    a = max(ids[:-1], key=p.ctx_len)
                    p.fork([a], [ids[-1]], [p.ctx_len(a) // P * P])
            except cpl.CrossPoolError as e:
                assert e.status == cpl.CP_ENOSPC
        elif not ids:
            continue
        elif op < 0.5:
            r = rng.choice(ids)
            grow(p, r, rng.randint(0, reserve * P - p.ctx_len(r)))
        elif op < 0.65 and len(ids) > 1:
            a, b = rng.sample(ids, 2)
            if p.ctx_len(b) == 0:
                p.fork([a], [b], [p.ctx_len(a) // P * P])
        elif op < 0.7:
            p.close(ids.pop(rng.randrange(len(ids))))
        else:
            some = rng.sample(ids, rng.randint(1, len(ids)))
            n = {r: p.ctx_len(r) for r in some}
            first = [rng.randint(0, n[r]) if rng.random() < 0.5 else 0 for r in some]
            lists = {r: sorted(rng.sample(range(n[r] - f), rng.randint(0, n[r] - f))) if rng.random() < 0.6 else
                     list(range(rng.randint(0, n[r] - f))) for r, f in zip(some, first)}
            pages, before = {r: p.pages(r).tolist() for r in ids}, p.stats()
            after, beside = cut_books(pages, reserve, first, lists)
            try:
                p.keep(some, first, [len(x) for x in lists.values()], [t for x in lists.values() for t in x])
                assert max(after, beside) <= total and p.stats()["pages_reserved"] == after
                together += len(some) > 1 and before["pages_used"] < sum(map(len, pages.values()))
            except cpl.CrossPoolError as e:
                assert e.status == cpl.CP_ENOSPC and max(after, beside) > total
                assert (p.stats(), {r: p.pages(r).tolist() for r in ids}) == (before, pages)
                refused += 1
    for r in ids:  # what was admitted can be filled
        grow(p, r, reserve * P - p.ctx_len(r))
    for r in ids:
        p.close(r)
    assert p.stats()["pages_used"] == p.stats()["pages_reserved"] == 0
    p.destroy()
    return refused, together


# ------------------------------------- rows per token in one another's memory

ROWS = """
import random, time
T = 16
def books(n, layers, heads):
    p = cpl.Pool(page_tokens=P, pool_bytes=4 << 30, chunk_bytes=1 << 20, device=0)
    m = p.register(cpl.CP_KIND_GQA, heads, heads, head_dim=64, n_layers=layers)
    ids = [p.open(m, T) for _ in range(n)]
    p.append(ids, [T] * n, at, 0)
    return p, ids
def weights(p, ids, layer, old, new):
    n = len(ids)
    return LIB.cp_attn_weights(p.handle, n, I32(*ids), I32(*[0] * n), None, None, layer, 0.5, old, new, None, None)
def evict(p, ids, w, new, kept):  # of nothing: requests are left as they are
    n = len(ids)
    o = cp_evict_opts(0, 0, *(None if x is None else ctypes.addressof(x) for x in (new, kept)))
    return LIB.cp_kv_evict(p.handle, n, I32(*ids), I64(*[T] * n), w, by(o), None)
BASE = 1 << 30
"""


def test_overlaps_of_rows_against_every_pair(queued):
    """Records of all kinds in a small memory: a call is refused where a row that it writes
    has an element of another's, but for sums in the place of their own old ones."""
    run(MORE + ROWS + """
rng = random.Random(7)
tally = {}
for layers, heads in ((1, 1), (1, 3), (2, 1), (3, 2)):
    p, ids = books(4, layers, heads)
    for trial in range(1500):
        n = rng.randint(1, 4)
        grid = rng.random() < 0.6  # one layout for all, or each its own
        def strides():
            head = rng.choice([T, T + 3, 2 * T, 4 * T, 5 * T])
            one = (heads - 1) * head + T
            return head, rng.choice([one, one + 5, one + T, 4 * heads * T, 8 * heads * T])
        shared = strides()
        def record():
            head, layer = shared if grid else strides()
            longest = min(head if heads > 1 else 99, layer - (heads - 1) * head if layers > 1 else 99)
            length = T if rng.random() < 0.7 else rng.randint(T, max(T, min(longest, T + 6)))
            start = rng.randrange(64) * T if rng.random() < 0.8 else rng.randrange(64 * T)
            return cp_token_rows(BASE + 4 * start, length, head, max(layer, (heads - 1) * head + length))
        first, second, third = ([record() for _ in range(n)] for _ in range(3))
        for i in range(n):
            if rng.random() < 0.6:
                x = first[i]
                second[i] = cp_token_rows(x.data, x.len if rng.random() < 0.8 else T, x.head, x.layer)
        third = third if rng.random() < 0.3 else None
        of_layer = rng.randrange(layers)
        for call in ("weights", "evict"):
            some = [of_layer] if call == "weights" else range(layers)
            cells = []  # (argument, entry, element, row)
            for a, recs in enumerate((first, second, third if call == "evict" else None)):
                for i, x in enumerate(recs or ()):
                    for l in some:
                        for h in range(heads):
                            at0 = (x.data - BASE) // 4 + (l * x.layer if layers > 1 else 0) + (h * x.head if heads > 1 else 0)
                            cells += [(a, i, at0 + t) for t in range(x.len)]
            def same(i):
                x, y = first[i], second[i]
                return x.data + (4 * of_layer * (x.layer - y.layer) if call == "weights" and layers > 1 else 0) == y.data and (
                    heads == 1 or x.head == y.head) and (call == "weights" or layers == 1 or x.layer == y.layer)
            by_cell, clash = {}, False
            for a, i, c in cells:
                for b, j in by_cell.setdefault(c, []):
                    if a == b == 0 or (a + b == 1 and i == j and same(i)):
                        continue
                    clash = True
                by_cell[c].append((a, i))
            if call == "weights":
                rc = weights(p, ids[:n], of_layer, rows(*first), rows(*second))
            else:
                rc = evict(p, ids[:n], rows(*first), rows(*second), rows(*third) if third else None)
            text = LIB.cp_last_error().decode()
            assert rc == (cpl.CP_EINVAL if clash else cpl.CP_OK), (rc, text, clash, trial, call, layers, heads)
            assert not clash or "overlap without being the same" in text
            tally[call, clash] = tally.get((call, clash), 0) + 1
    for r in ids:
        p.close(r)
    p.destroy()
assert min(tally.values()) > 800 and len(tally) == 4, tally
""", queued)


LAYOUTS = {  # (start, from head to head, from layer to layer) of request r's rows, in one tensor
    "[layer][request][head][token]": "(r * H * T, T, n * H * T)",
    "[layer][head][request][token]": "(r * T, n * T, n * H * T)",
    "[request][layer][head][token]": "(r * n_layers * H * T, T, H * T)",
    "half of the requests each way": "(r * T, n * T // 2, n * H * T) if r < n // 2 else (r * H * T, T, n * H * T)",
    "layers apart by the request": "(r * T, 2 * n * T, 2 * n * H * T + r)",
}


@pytest.mark.parametrize("layout", sorted(LAYOUTS))
def test_many_requests_in_one_tensor_are_looked_through_once(layout, queued):
    """512 requests of 16 layers and 8 KV heads (a second and more where every pair of
    requests was compared, row by row)."""
    run(MORE + ROWS + f"""
n, n_layers, H = 512, 16, 8
place = lambda r: {LAYOUTS[layout]}
p, ids = books(n, n_layers, H)
recs = [cp_token_rows(BASE + 4 * a, T, h, l) for a, h, l in map(place, range(n))]
W = rows(*recs)
t0 = time.perf_counter()
assert evict(p, ids, W, W, None) == cpl.CP_OK, LIB.cp_last_error()
assert weights(p, ids, 3, W, W) == cpl.CP_OK
took = time.perf_counter() - t0
assert took < 0.5, took
x = recs[200]
recs[200] = cp_token_rows(x.data + 4, x.len, x.head, x.layer)  # some last element is another's first
assert evict(p, ids, rows(*recs), rows(*recs), None) == cpl.CP_EINVAL
for r in ids:
    p.close(r)
p.destroy()
""", queued)


def test_an_eviction_of_no_request(queued):
    """Empty lists of rows are of either type."""
    run(MORE + """
p, m = heads_pool()
p.evict([], [], [], 0, new=[], kept=[])
none = cpl.token_rows([])
p.evict([], [], none, 0, new=none, kept=none)
p.destroy()
""", queued)
