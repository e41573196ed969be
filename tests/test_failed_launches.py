"""Launches that fail after a call has changed the pool's tables (CPU: the HIP
runtime is a stand-in whose n-th launch or copy fails). The pool refuses further
work on its device memory, whose page table is behind the host's, and can
still be closed; a call that fails before that leaves it as it was."""
import os
import shutil
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))

SETUP = """
import ctypes, sys
sys.modules["torch"] = None
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
from paper_2606_24506_amd import crosspool as cpl

P = 4
mem = (ctypes.c_char * (1 << 16))()
at = (ctypes.addressof(mem) + 255) // 256 * 256  # (kernels do not run: nothing is read there)

def pool(layers=1, **kw):
    p = cpl.Pool(page_tokens=P, pool_bytes=8 << 20, chunk_bytes=1 << 14, device=0, **kw)
    return p, p.register(cpl.CP_KIND_GQA, 2, 1, head_dim=64, n_layers=layers)

def status(fn, *args, **kw):
    try:
        fn(*args, **kw)
    except cpl.CrossPoolError as e:
        return e.status, str(e)
    return cpl.CP_OK, ""

def unusable(p, ids, m):
    a = ids[0]
    other = p.open(m, 8)
    for fn, args in ((p.append, ([a], [1], at, 0)), (p.decode, ([a], at, at, at, 0)), (p.gather, (a, 0, 1, at, 0)),
                     (p.decode_step, ([a], [1], at, at, at, at, 0)), (p.extend, ([a], [1], at, at, at, 0)),
                     (p.extend_step, ([a], [1], at, at, at, at, 0)), (p.fork, ([a], [other], None, 0)),
                     (p.truncate, ([a], [0], 0))):
        rc, text = status(fn, *args)
        assert rc == cpl.CP_ESTATE and "destroy" in text, (fn, rc, text)
    for r in (*ids, other):
        p.close(r)
    p.destroy()

def usable(p, ids):
    before = p.stats()
    q = p.open(0, 8)
    p.fork([ids[0]], [q], [P], 0)
    p.extend([q], [1], at, at, at, 0)
    p.gather(q, 0, P, at, 0)
    p.close(q)
    assert p.stats() == before
    for r in ids:
        p.close(r)
    p.destroy()
"""

CASES = {
    "fork": """
p, m = pool()
a, b = p.open(m, 40), p.open(m, 40)
p.append([a], [10], at, 0)
fake.fake_fail_in(1)
assert status(p.fork, [a], [b], None, 0)[0] == cpl.CP_EHIP
unusable(p, [b, a], m)
""",
    "fork of many planes, the second launch": """
p, m = pool(layers=70)
a, b = p.open(m, 40), p.open(m, 40)
p.append([a], [10], at, 0)
fake.fake_fail_in(2)
assert status(p.fork, [a], [b], None, 0)[0] == cpl.CP_EHIP
unusable(p, [a, b], m)
""",
    "truncate inside a shared page": """
p, m = pool()
a, b = p.open(m, 40), p.open(m, 40)
p.append([a], [12], at, 0)
p.fork([a], [b], None, 0)
fake.fake_fail_in(1)
assert status(p.truncate, [b], [6], 0)[0] == cpl.CP_EHIP
unusable(p, [b, a], m)
""",
    "step, the append": """
p, m = pool()
a = p.open(m, 40)
p.append([a], [10], at, 0)
fake.fake_fail_in(1)
assert status(p.extend_step, [a], [3], at, at, at, at, 0)[0] == cpl.CP_EHIP
unusable(p, [a], m)
""",
    "step, the page-table copy": """
p, m = pool(layers=3)
a = p.open(m, 40)
fake.fake_fail_in(1)
launches = fake.fake_launches()
assert status(p.extend_step, [a], [9], at, at, at, at, 0)[0] == cpl.CP_EHIP
assert fake.fake_launches() == launches
unusable(p, [a], m)
""",
    "step, the attention": """
p, m = pool()
a = p.open(m, 40)
p.append([a], [10], at, 0)
fake.fake_fail_in(2)
assert status(p.extend_step, [a], [3], at, at, at, at, 0)[0] == cpl.CP_EHIP
unusable(p, [a], m)
""",
    "attention alone changes nothing": """
p, m = pool()
a = p.open(m, 40)
p.append([a], [10], at, 0)
fake.fake_fail_in(1)
assert status(p.extend, [a], [3], at, at, at, 0)[0] == cpl.CP_EHIP
usable(p, [a])
""",
    "no memory for the workspace": """
p, m = pool()
a = p.open(m, 400)
p.append([a], [400], at, 0)
fake.fake_no_memory(1)
assert status(p.extend_step, [a], [0], at, at, at, at, 0)[0] == cpl.CP_OK
assert status(p.extend, [a], [8], at, at, at, 0, num_splits=3)[0] == cpl.CP_ENOMEM
assert status(cpl.Rope, 8)[0] == status(pool)[0] == cpl.CP_ENOMEM
b = p.open(m, 40)
p.fork([a], [b], [6], 0)  # (and no launch reports the allocation)
fake.fake_no_memory(0)
p.close(b)
usable(p, [a])
""",
    "an error left behind by another call": """
p, m = pool()
a, b = p.open(m, 40), p.open(m, 40)
p.append([a], [12], at, 0)
before = p.stats()
for fn, args in ((p.fork, ([a], [b], None, 0)), (p.extend_step, ([a], [3], at, at, at, at, 0))):
    fake.fake_leave_error(1)  # an invalid value
    assert status(fn, *args)[0] == cpl.CP_EHIP
    assert p.stats() == before and (p.ctx_len(a), p.ctx_len(b)) == (12, 0)
p.fork([a], [b], None, 0)
fake.fake_leave_error(1)  # an invalid value
assert status(p.truncate, [b], [6], 0)[0] == cpl.CP_EHIP
assert p.ctx_len(b) == 12
fake.fake_leave_error(600)  # an event that is not ready
p.truncate([b], [6], 0)
fake.fake_leave_error(600)
p.extend_step([a], [3], at, at, at, at, 0)
usable(p, [a, b])
""",
}


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    out = str(tmp_path_factory.mktemp("fake") / "fake_hip.so")
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", os.path.join(HERE, "c", "fake_hip.cpp"), "-o", out], check=True)
    return out


@pytest.mark.parametrize("case", sorted(CASES))
def test_failures_after_the_tables_changed(case, fake):
    res = subprocess.run([sys.executable, "-c", SETUP + CASES[case], fake], cwd=os.path.dirname(HERE), capture_output=True,
                         text=True, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
