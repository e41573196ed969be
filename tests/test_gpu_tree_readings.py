"""Drafted trees beside the calls that they lead to: a chain deeper than its sliding
window, whose masks the caller limits, is the chunk that cp_attn_extend attends; and
the weights that the accepted path gives are of its own queries, packed."""
import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import Scene, attend, check, rounds_to_16_bits
from test_gpu_tree import device_tree
from test_gpu_weights import compare
from token_ref import ancestors, given, make_tree, pack

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mqa32d128", "gqa4x2d256", "mla16"])
@pytest.mark.parametrize("n, window", [(3, 2), (7, 1), (40, 9), (150, 40), (150, 149)])
def test_a_chain_deeper_than_its_window_with_masks_of_the_callers(name, n, window):
    """cp_tree_build names every ancestor, and the window does not reach into a tree: an
    ancestor `window` or more positions back goes out of the mask."""
    print(f"[case] chain {name} {n} window {window}", flush=True)
    sc = Scene(name, [n, n + 70, 333], seed=11)
    parents = [list(range(-1, n - 1))] * 3
    mask, depth = device_tree(parents)
    t, u = torch.arange(n)[:, None], torch.arange(n)[None]
    near = pack((u <= t) & (u > t - window), mask.shape[1]).cuda()
    q, out, lse = sc.buffers(3 * n)
    sc.pool.tree(sc.ids, [n] * 3, q, out, lse, mask & near.repeat(3, 1), depth, window=window)
    for i, rows in enumerate(sc.rows):
        part = slice(n * i, n * i + n)
        check(out[part], lse[part], attend(name, rows, q[part], window=window), rounds_to_16_bits(name, n),
              f"{name} chain {i}")
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("size", [9, 90])
def test_weights_of_an_accepted_path(name, size):
    """Behind cp_request_keep the path's tokens are the context's last, and saw what a chunk
    of them sees: their q and lse, packed, are those that cp_attn_weights takes."""
    print(f"[case] path's weights {name} {size}", flush=True)
    held = [180, 5, 700]
    sc = Scene(name, held, seed=12, room=100)
    trees = [make_tree(size, 1, width=2, roots=0.02), make_tree(size, 2, width=3), make_tree(1, 3)]
    sizes = [len(t) for t in trees]
    mask, depth = device_tree(trees)
    new = sc.normal(sum(sizes), sc.row, sigma=0.7)
    q, out, lse = sc.buffers(sum(sizes))
    sc.pool.tree_step(sc.ids, sizes, new, q, out, lse, mask, depth)
    paths = [ancestors(t)[0][len(t) - 1].nonzero()[:, 0].tolist() for t in trees]
    sc.pool.keep(sc.ids, held, [len(p) for p in paths], sum(paths, []))
    at = [sum(sizes[:i]) + k for i, p in enumerate(paths) for k in p]
    q, lse = q[at].contiguous(), lse[at].contiguous()
    sums = [torch.rand(sc.hkv, n + len(p), device="cuda") for n, p in zip(held, paths)]
    old = [s.clone() for s in sums]
    sc.pool.weights(sc.ids, [len(p) for p in paths], q, lse, sums, old=sums, decay=0.5)
    k = 0
    for i, p in enumerate(paths):
        rows = sc.held(sc.ids[i], held[i] + len(p))
        part = slice(k, k + len(p))
        compare(sums[i], given(name, rows, q[part], lse[part]), old[i], 0.5, f"{name} request {i}")
        check(out[at][part], lse[part], attend(name, rows, q[part]), rounds_to_16_bits(name, sizes[i]), f"{name} path {i}")
        k += len(p)
    sc.close()
