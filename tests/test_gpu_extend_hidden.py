"""Large finite values of V in attention of token chunks: out of a row's sight
they add nothing to it, however large, and in sight no more than their weight."""
import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, Scene, attend, check, rounds_to_16_bits, shape

pytestmark = pytest.mark.gpu

LARGEST = torch.finfo(torch.bfloat16).max  # 3.39e38


def v_columns(name):
    hq, hkv, dk, dv, row, _ = shape(name)
    return slice(0, dv) if GEOMS[name]["kind"] == cpl.CP_KIND_MLA else slice(hkv * dk, row)


def run(sc, n_q, q=None, **opts):
    q = sc.buffers(n_q)[0] if q is None else q
    _, out, lse = sc.buffers(n_q)
    sc.pool.extend(sc.ids[:1], [n_q], q, out, lse, **opts)
    torch.cuda.synchronize()
    return q, out, lse


def replace(sc, rows):
    sc.pool.truncate(sc.ids[:1], [0])
    sc.pool.append(sc.ids[:1], [rows.shape[0]], rows)


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mha3d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("n_q", [2, 3, 6, 40])
@pytest.mark.parametrize("value", [LARGEST, -LARGEST, 1e36])
@pytest.mark.parametrize("by", ["causality", "documents", "window"])
def test_large_values_out_of_sight_add_nothing(name, n_q, value, by):
    """One token's V is large; the rows that do not see it are as if it were not
    there (those that do see it are not looked at)."""
    print(f"[case] extend large {name} {n_q} {value} {by}", flush=True)
    n = 150
    first = n - n_q  # position of the first row
    sc = Scene(name, [n], seed=40)
    # seen by at least one row, so that its tile reads it, and hidden from another
    where = {"causality": n - 1, "documents": 60, "window": first - 20}[by]
    rows = sc.rows[0].clone()
    rows[where, v_columns(name)] = value
    replace(sc, rows)
    opts = {}
    sees = torch.arange(first, n) >= where
    if by == "documents":
        opts["doc_begin"] = torch.tensor([61 if i else 0 for i in range(n_q)], dtype=torch.int32, device="cuda")
        sees = torch.arange(n_q) == 0
    elif by == "window":
        opts["window"] = 21  # the first row sees `where` as its last
        sees = torch.arange(n_q) == 0
    q, out, lse = run(sc, n_q, **opts)
    clean = rows.clone()
    clean[where] = 0
    ref = attend(name, clean, q, **opts)
    assert 0 < int((~sees).sum()) < n_q
    check(out[~sees.cuda()], lse[~sees.cuda()], tuple(x[~sees] for x in ref), rounds_to_16_bits(name, n_q), f"{name} {by}")
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("n_q", [1, 6])
@pytest.mark.parametrize("n", [128, 256])
def test_large_values_in_sight_weigh_what_they_weigh(name, n_q, n):
    """A key whose score is about 100 below the others: e^-100 1e38 is nothing."""
    print(f"[case] extend weight {name} {n_q} {n}", flush=True)
    sc = Scene(name, [n + n_q - 1], seed=41)
    hq, hkv, dk, dv, row, scale = shape(name)
    rows = sc.rows[0].clone()
    mla = GEOMS[name]["kind"] == cpl.CP_KIND_MLA
    q = sc.buffers(n_q)[0]
    # one K element that V does not hold (MLA: of the rotary part) makes the score
    e = dv if mla else 0
    q[..., e] = 16.0
    low = -100 / (16.0 * scale)
    rows[:, v_columns(name)] = sc.normal(rows.shape[0], row)[:, v_columns(name)]
    for c in range(1 if mla else hkv):
        rows[:, c * dk + e] = 0
        rows[40, c * dk + e] = low
    rows[40, v_columns(name)] = 1e38
    if mla:  # its latent part makes scores too: none
        q[..., :dv] = 0
    replace(sc, rows)
    q, out, lse = run(sc, n_q, q=q)
    check(out, lse, attend(name, rows, q), rounds_to_16_bits(name, n_q), f"{name}")
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "gqa4x2d256"])
@pytest.mark.parametrize("n_q", [1, 6, 40])
@pytest.mark.parametrize("n,low,splits", [(128, 32, 1), (600, 200, 3), (3000, 1500, 23)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_special_values_in_sight_are_not_lost_in_joins(name, n_q, n, low, splits, bad):
    """NaN in a V that a row sees gives NaN there, an infinite one no finite
    result, also where all keys around it weigh nothing (their scores are 400
    below the others) and their sums join those of the rest with weight 0."""
    print(f"[case] extend lost {name} {n_q} {n} {splits} {bad}", flush=True)
    sc = Scene(name, [n + n_q - 1], seed=42)
    hq, hkv, dk, dv, row, scale = shape(name)
    rows = sc.rows[0].clone()
    q = sc.buffers(n_q)[0]
    q[..., 0] = 16.0
    for c in range(hkv):
        rows[:low, c * dk] = -400 / (16.0 * scale)
        rows[low:, c * dk] = 0
    rows[20, hkv * dk + 5] = bad
    replace(sc, rows)
    _, out, _ = run(sc, n_q, q=q, num_splits=splits)
    got = out[:, :hq // hkv, 5]
    assert torch.isnan(got).all() if bad != bad else not torch.isfinite(got).any()
    out[:, :hq // hkv, 5] = 0
    assert torch.isfinite(out).all()
    sc.close()
