"""The precision of a request's chunk attention is its own: beside other requests, and
beside branches whose pages it shares, it gets the probabilities that it gets alone."""
import pytest
import torch

from prompt_ref import Scene, attend, check, rounds_to_16_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mqa32d128", "mha3d64", "gqa4x2d256"])
@pytest.mark.parametrize("n_q", [[1] * 20, [1, 3, 1, 1, 2, 6, 1, 1], [2] * 5 + [60, 1, 1], [40, 33]])
@pytest.mark.parametrize("shared", [512, 4000])
def test_branches_keep_their_precision(name, n_q, shared):
    """Peaked scores, so that a probability's rounding shows in columns where the
    sum of p V is small beside that of p |V|."""
    print(f"[case] extend company {name} {n_q} {shared}", flush=True)
    sc = Scene(name, [shared], seed=50, room=100, pool_bytes=256 << 20)
    parent = sc.ids[0]
    kids, rows = [], []
    for i, k in enumerate(n_q):
        rid = sc.pool.open(sc.model, shared + 100)
        sc.pool.fork([parent], [rid])
        tail = sc.normal(k + i % 3, sc.row, sigma=0.7)
        sc.pool.append([rid], [k + i % 3], tail)
        kids.append(rid)
        rows.append(torch.cat([sc.rows[0], tail]))
    q, out, lse = sc.buffers(sum(n_q))
    q *= 4
    sc.pool.extend(kids, n_q, q, out, lse)
    torch.cuda.synchronize()
    at = 0
    for i, k in enumerate(n_q):
        check(out[at:at + k], lse[at:at + k], attend(name, rows[i], q[at:at + k]), rounds_to_16_bits(name, k),
              f"{name} branch {i}")
        at += k
    sc.ids += kids
    sc.close()
