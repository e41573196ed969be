"""Capped scores of chunk attention by themselves: with a window of one token a
row's lse is its own capped score."""
import math

import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, Scene, shape

pytestmark = pytest.mark.gpu


def capped(sc, q_value, k_value, cap, path=cpl.CP_PATH_AUTO):
    """lse [tokens][heads] of rows whose product is q_value * k_value."""
    n = q_value.shape[0]
    mla = GEOMS[sc.name]["kind"] == cpl.CP_KIND_MLA
    e = sc.dv if mla else 0
    rows = torch.zeros(n, sc.row, dtype=torch.bfloat16, device="cuda")
    for c in range(1 if mla else sc.hkv):
        rows[:, c * sc.dk + e] = k_value
    sc.pool.truncate(sc.ids, [0])
    sc.pool.append(sc.ids, [n], rows)
    q, out, lse = sc.buffers(n)
    q.zero_()
    q[..., e] = q_value
    sc.pool.extend(sc.ids, [n], q, out, lse, softcap=cap, window=1, path=path)
    torch.cuda.synchronize()
    return lse.double().cpu()


@pytest.mark.parametrize("name,path", [("gqa8x2d128", cpl.CP_PATH_AUTO), ("gqa6x2d64", cpl.CP_PATH_AUTO),
                                       ("mla16", cpl.CP_PATH_AUTO), ("gqa8x2d128", cpl.CP_PATH_VALU)])
@pytest.mark.parametrize("n", [2, 6, 400])
@pytest.mark.parametrize("cap", [0.5, 50.0])
@pytest.mark.parametrize("spread", [False, True])
def test_capped_scores_against_64_bits(name, path, n, cap, spread):
    """Arguments from 1e-3 to 9, sorted (waves of small ones alone) and mixed. The
    tangent is good to 7e-7 of its value; the argument is rounded three times
    and the result four (2^-24 each, and the tangent's argument counts at most once);
    the logarithm of a sum of one adds 2^-22."""
    print(f"[case] caps {name} {path} {n} {cap} {spread}", flush=True)
    sc = Scene(name, [0], seed=60, room=n)
    hq, _, _, _, _, scale = shape(name)
    worst = 0.0
    for part in range(max(1, 400 // n) if n < 400 else 1):
        count = n * hq
        x = torch.logspace(-3, math.log10(9), 400 * hq, dtype=torch.float64)[part * count:(part + 1) * count]
        x[1::2] *= -1
        if spread:
            x = x[torch.randperm(count, generator=torch.Generator().manual_seed(part))]
        q = (x * cap / scale).view(n, hq).to(torch.bfloat16)
        want = cap * torch.tanh(q.double() * scale / cap)
        got = capped(sc, q.cuda(), 1.0, cap, path)
        worst = max(worst, ((got - want).abs() / ((7e-7 + 7 * 2.0 ** -24) * want.abs() + 2.0 ** -22)).max().item())
    print(f"[caps] {worst:.3f} of the tolerance", flush=True)
    assert worst <= 1
    sc.close()


@pytest.mark.parametrize("n", [2, 12, 40])
@pytest.mark.parametrize("path", [cpl.CP_PATH_AUTO, cpl.CP_PATH_VALU])
def test_products_whose_squares_pass_32_bits(n, path):
    """Products of 2^58 to 2^64 under a cap of 1e18, with a small scale: arguments
    of the tangent far under 1, whose products' squares pass 2^128."""
    GEOMS["small scale"] = dict(kind=cpl.CP_KIND_GQA, n_q_heads=4, n_kv_heads=2, head_dim=64, softmax_scale=0.01)
    try:
        sc = Scene("small scale", [0], seed=61, room=n)
        q = 2.0 ** (28 + torch.arange(4 * n).view(n, 4) % 7)
        got = capped(sc, q.to(torch.bfloat16).cuda(), 2.0 ** 30, 1e18, path)
        want = 1e18 * torch.tanh(q.double() * 2.0 ** 30 * 0.01 / 1e18)
        assert ((got - want).abs() <= 2e-6 * want.abs()).all(), (got, want)
        sc.close()
    finally:
        del GEOMS["small scale"]
