"""Requests cut to some of their tokens, on the CPU: what a call does that its
neighbours in the call, earlier work of the stream or its size could change (a
stand-in for the HIP runtime, tests/c/queued_hip.cpp, or a host-only pool)."""
import os
import shutil
import subprocess

import pytest

from paper_2606_24506_amd import build
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
