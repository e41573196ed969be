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
