"""Attention of token chunks over the pool (cp_attn_extend) against the 64-bit
form: geometries, page sizes, lengths from one token on, every mask and their
combinations, rows that see nothing, infinities and NaN out of sight, ranges
joined, empty and ragged batches."""
import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, Scene, attend, check, rounds_to_16_bits, shape

pytestmark = pytest.mark.gpu


def run(sc, n_q, ids=None, q=None, **opts):
    ids = sc.ids if ids is None else ids
    total = sum(n_q)
    buf = sc.buffers(total)
    q = buf[0] if q is None else q
    sc.pool.extend(ids, n_q, q, buf[1], buf[2], **opts)
    torch.cuda.synchronize()
    return q, buf[1], buf[2]


def verify(sc, n_q, label, rows=None, together=False, **opts):
    """together: rows of several requests share tiles, of more than 32 rows, whose
    probabilities are rounded to bf16 (off by at most 2^-8 of themselves)."""
    q, out, lse = run(sc, n_q, **opts)
    at = 0
    path = opts.pop("path", cpl.CP_PATH_AUTO)
    opts.pop("num_splits", None)
    prefix, docs = opts.pop("prefix", None), opts.pop("doc_begin", None)
    for i, k in enumerate(n_q):
        if k == 0:
            continue
        ref = attend(sc.name, (rows or sc.rows)[i], q[at:at + k], prefix=prefix[i] if prefix else 0,
                     doc_begin=docs[at:at + k] if docs is not None else None, **opts)
        check(out[at:at + k], lse[at:at + k], ref, together or rounds_to_16_bits(sc.name, k, path), f"{label} request {i}")
        at += k


@pytest.mark.parametrize("name", sorted(GEOMS))
@pytest.mark.parametrize("path", [cpl.CP_PATH_AUTO, cpl.CP_PATH_VALU])
def test_causal_chunks_of_every_geometry(name, path):
    """One token, a few, and chunks past a tile, some being the whole context."""
    print(f"[case] extend {name} path {path}", flush=True)
    sc = Scene(name, [1, 63, 200, 129, 300], seed=3)
    verify(sc, [1, 1, 7, 129, 70], f"{name} path {path}", path=path)
    verify(sc, [0, 3, 0, 1, 2], f"{name} path {path}", path=path)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("page_tokens", [1, 6, 16, 48, 150])
def test_page_sizes(name, page_tokens):
    if page_tokens * 2 * shape(name)[4] % 256:
        pytest.skip("pages of this model are no multiple of 256 bytes")
    print(f"[case] extend pages {name} {page_tokens}", flush=True)
    sc = Scene(name, [77, 310], page_tokens=page_tokens, seed=4)
    verify(sc, [1, 60], f"{name} P{page_tokens}")
    sc.close()


MASKS = {
    "cap": dict(softcap=3.0),
    "weak cap": dict(softcap=50.0),
    "slopes": dict(slopes=True),
    "window": dict(window=37),
    "window 1": dict(window=1),
    "prefix": dict(prefix=[150, 1000, 0]),
    "docs": dict(docs=True),
    "all": dict(softcap=5.0, slopes=True, window=90, prefix=[180, 0, 40], docs=True),
}


@pytest.mark.parametrize("mask", sorted(MASKS))
@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mqa32d128", "mla20", "mla4l128r40"])
@pytest.mark.parametrize("n_q", [[1, 1, 1], [4, 2, 5], [130, 61, 33]])
def test_masks(mask, name, n_q):
    print(f"[case] extend mask {mask} {name} {n_q}", flush=True)
    sc = Scene(name, [201, 130, 67], seed=5)
    opts = dict(MASKS[mask])
    if opts.pop("slopes", None):
        opts["slopes"] = torch.linspace(0.5, 0.01, sc.hq, device="cuda")
    if opts.pop("docs", None):
        starts = []
        for n, k in zip([201, 130, 67], n_q):
            starts += [max(0, (p // 23) * 23 - 5) for p in range(n - k, n)]
        opts["doc_begin"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    verify(sc, n_q, f"{mask} {name}", **opts)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l64r0"])
@pytest.mark.parametrize("n_q", [2, 40])
@pytest.mark.parametrize("splits", [0, 3])
def test_rows_that_see_nothing(name, n_q, splits):
    """Documents that start behind a token leave its row empty: some rows, and all."""
    print(f"[case] extend empty {name} {n_q} {splits}", flush=True)
    sc = Scene(name, [300], seed=6)
    some = torch.tensor([300 if i % 3 == 0 else -7 for i in range(n_q)], dtype=torch.int32, device="cuda")
    verify(sc, [n_q], f"{name} some", doc_begin=some, num_splits=splits)
    none = torch.full((n_q,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    verify(sc, [n_q], f"{name} none", doc_begin=none, num_splits=splits)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mqa32d128", "mla16", "mla128", "gqa4x2d256"])
@pytest.mark.parametrize("splits", [2, 5, 64])
@pytest.mark.parametrize("n_q", [1, 50])
def test_ranges_are_joined(name, splits, n_q):
    print(f"[case] extend splits {name} {splits} {n_q}", flush=True)
    sc = Scene(name, [1500, 65], seed=7)
    verify(sc, [n_q, min(n_q, 65)], f"{name} splits {splits}", num_splits=splits)
    verify(sc, [n_q, min(n_q, 65)], f"{name} splits {splits} window", num_splits=splits, window=100)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("n_q", [1, 3, 90])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_special_values_out_of_sight_stay_there(name, n_q, bad):
    """Keys and values that a row does not see (outside its window or
    document, after it, or stale memory past the context) do not reach it; a
    row that sees an infinite value gets it."""
    print(f"[case] extend special {name} {n_q} {bad}", flush=True)
    n = 210
    sc = Scene(name, [n], seed=8, fill=float("nan"), page_tokens=64)
    hq, hkv, dk, dv, row, _ = shape(name)
    rows = sc.rows[0].clone()
    where = n - n_q // 2 - 1 if n_q > 1 else 100
    rows[where, :] = bad  # one token's K and V
    sc.pool.truncate([sc.ids[0]], [0])
    sc.pool.append([sc.ids[0]], [n], rows)
    # rows before `where` do not see it (causal), rows after only look behind it
    starts = torch.tensor([0 if p < where else where + 1 for p in range(n - n_q, n)], dtype=torch.int32, device="cuda")
    q, out, lse = run(sc, [n_q], doc_begin=starts)
    clean = rows.clone()
    clean[where] = 0
    ref = attend(name, clean, q, doc_begin=starts)
    check(out, lse, ref, rounds_to_16_bits(name, n_q), f"{name} {bad}")
    # only one element of V is special: the rows that see it have it, in that column alone
    if GEOMS[name]["kind"] == cpl.CP_KIND_GQA and bad == bad:
        rows = sc.rows[0].clone()
        rows[where, hkv * dk + 5] = bad
        sc.pool.truncate([sc.ids[0]], [where])
        sc.pool.append([sc.ids[0]], [n - where], rows[where:].contiguous())
        q, out, lse = run(sc, [n_q])
        sees = torch.arange(n - n_q, n) >= where
        g = hq // hkv
        got = out.float().cpu()
        assert torch.equal(got[sees][:, :g, 5], torch.full((int(sees.sum()), g), bad))
        assert torch.isfinite(got[~sees]).all()
        got[:, :g, 5] = 0
        assert torch.isfinite(got).all()
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "mla16"])
@pytest.mark.parametrize("n_q", [1, 40])
def test_nan_scores_in_sight_give_nan(name, n_q):
    sc = Scene(name, [100], seed=9)
    q = sc.buffers(n_q)[0]
    q[0, 0] = float("nan")
    _, out, lse = run(sc, [n_q], q=q)
    assert torch.isnan(out[0, 0]).all() and torch.isnan(lse[0, 0])
    assert torch.isfinite(out[0, 1:]).all() and torch.isfinite(out[1:]).all()
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16"])
def test_one_token_equals_decode(name):
    """Causal attention of the last token is what the decode call computes."""
    sc = Scene(name, [1, 64, 1000, 4097], seed=10)
    q, out, lse = run(sc, [1] * 4)
    o2, l2 = torch.zeros_like(out), torch.zeros_like(lse)
    sc.pool.decode(sc.ids, q, o2, l2)
    torch.cuda.synchronize()
    assert torch.allclose(lse, l2, atol=1e-4)
    # each off by half a step, and decode's probabilities too
    assert ((out.float() - o2.float()).abs() <= 2.0 ** -7 * out.float().abs() + 2.0 ** -7 * 0.7 * 4).all()
    sc.close()


def test_results_do_not_depend_on_placement_or_company():
    """The same request alone on other pages: the same bits."""
    sc = Scene("gqa8x2d128", [700, 300, 50], seed=11)
    q, out, lse = run(sc, [65, 3, 1], num_splits=3)
    pool = cpl.Pool(page_tokens=64, pool_bytes=64 << 20, placement_seed=99, device=0)
    m = pool.register(**GEOMS["gqa8x2d128"])
    rid = pool.open(m, 700)
    pool.append([rid], [700], sc.rows[0])
    o2, l2 = torch.zeros_like(out[:65]), torch.zeros_like(lse[:65])
    pool.extend([rid], [65], q[:65].contiguous(), o2, l2, num_splits=3)
    torch.cuda.synchronize()
    assert torch.equal(o2, out[:65]) and torch.equal(l2, lse[:65])
    pool.close(rid)
    pool.destroy()
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("mask", ["causal", "all", "window"])
@pytest.mark.parametrize("shared,n_q", [(640, [1, 1, 1, 1, 1]), (1000, [3, 1, 5, 2, 9]), (300, [40, 1, 7, 2, 1])])
def test_forks_read_their_shared_pages_once(name, mask, shared, n_q):
    """Branches of one prompt, with tails and queries of different lengths, next
    to requests that share nothing; the same as with every request whole."""
    print(f"[case] extend shared {name} {mask} {shared} {n_q}", flush=True)
    sc = Scene(name, [shared], page_tokens=64, seed=15, room=100, pool_bytes=256 << 20)
    kids, rows = [], []
    for i, k in enumerate(n_q):
        rid = sc.pool.open(sc.model, shared + 400)
        keep = shared if i != 3 else shared - 70  # one shares less
        sc.pool.fork([sc.ids[0]], [rid], [keep])
        tail = sc.normal(k + 13 * i, sc.row, sigma=0.7)
        sc.pool.append([rid], [k + 13 * i], tail)
        kids.append(rid)
        rows.append(torch.cat([sc.rows[0][:keep], tail]))
    sc.add(100)
    ids = kids[:2] + [sc.ids[1]] + kids[2:]
    held = rows[:2] + [sc.rows[1]] + rows[2:]
    counts = n_q[:2] + [4] + n_q[2:]
    sc.ids = ids + [sc.ids[0]]
    sc.rows = held + [sc.rows[0]]
    counts.append(2)
    opts = {}
    if mask == "window":
        opts = dict(window=200)
    if mask == "all":
        opts = dict(softcap=8.0, window=500, prefix=[50, 0, 30, 5000, 0, 100, 7],
                    slopes=torch.linspace(0.3, 0.01, sc.hq, device="cuda"),
                    doc_begin=torch.tensor([(37 * i) % 260 for i in range(sum(counts))], dtype=torch.int32, device="cuda"))
    q, out, lse = run(sc, counts, **opts)
    q, o2, l2 = run(sc, counts, q=q, num_splits=1, **opts)
    at = 0
    more = {k: v for k, v in opts.items() if k not in ("prefix", "doc_begin")}
    for i, k in enumerate(counts):
        ref = attend(name, sc.rows[i], q[at:at + k], prefix=opts["prefix"][i] if "prefix" in opts else 0,
                     doc_begin=opts["doc_begin"][at:at + k] if "doc_begin" in opts else None, **more)
        check(out[at:at + k], lse[at:at + k], ref, True, f"{name} {mask} request {i}")  # (all rows together may be many)
        check(o2[at:at + k], l2[at:at + k], ref, True, f"{name} {mask} request {i} whole")
        at += k
    sc.close()


def test_many_branches_of_two_prompts():
    """More branches than a launch holds members of."""
    sc = Scene("gqa8x2d128", [500, 300], seed=16, room=10, pool_bytes=256 << 20)
    parents, base = list(sc.ids), list(sc.rows)
    ids, rows = [], []
    for p, n in ((0, 90), (1, 15)):
        kids = [sc.pool.open(sc.model, 600) for _ in range(n)]
        sc.pool.fork([parents[p]] * n, kids)
        tails = sc.normal(n, 2, sc.row, sigma=0.7)
        sc.pool.append(kids, [2] * n, tails)
        ids += kids
        rows += [torch.cat([base[p], t]) for t in tails]
    sc.ids, sc.rows = ids + parents, rows + base
    verify(sc, [1] * len(sc.ids), "105 branches", together=True)
    sc.close()


def test_many_requests_take_several_launches():
    lens = [1 + (37 * i) % 190 for i in range(150)]
    sc = Scene("gqa6x2d64", lens, seed=12)
    verify(sc, [min(n, 1 + i % 12) for i, n in enumerate(lens)], "150 requests")
    sc.close()


def test_more_joined_rows_than_one_launch_takes():
    """2^22 and some rows in two ranges: the join goes in parts, and gives what
    whole rows give (each side off by the roundings of its probabilities)."""
    n = (1 << 14) + 50
    pool = cpl.Pool(page_tokens=64, pool_bytes=64 << 20, device=0)
    m = pool.register(cpl.CP_KIND_GQA, 256, 1, head_dim=64)
    rid = pool.open(m, n)
    pool.append([rid], [n], torch.randn(n, 128, device="cuda").bfloat16())
    q = torch.randn(n, 256, 64, device="cuda").bfloat16()
    out, lse = torch.zeros_like(q), torch.zeros(n, 256, device="cuda")
    o2, l2 = torch.zeros_like(q), torch.zeros(n, 256, device="cuda")
    pool.extend([rid], [n], q, out, lse, num_splits=2, window=3000)
    pool.extend([rid], [n], q, o2, l2, num_splits=1, window=3000)
    torch.cuda.synchronize()
    assert torch.allclose(lse, l2, atol=1e-4)
    # outputs to half a step each, probabilities to 2^-8 of sums of p |v|, where |v| < 6
    assert ((out.float() - o2.float()).abs() <= 2.0 ** -7 * out.float().abs() + 2 * 2.0 ** -8 * 6).all()
    assert (out[-1].float() - o2[-1].float()).abs().max() < 0.02 and (o2[-1] != 0).any()
    pool.close(rid)
    pool.destroy()


def test_long_context_far_positions():
    """One row over 70001 tokens, planned ranges, slopes and a cap."""
    sc = Scene("gqa8x2d128", [70001], seed=13)
    verify(sc, [1], "long", slopes=torch.linspace(0.01, 1e-5, 8, device="cuda"), softcap=30.0)
    verify(sc, [9], "long window", window=65536)
    sc.close()


def test_graph_replays_and_streams():
    """Captured and replayed with eager calls between, on a stream of its own."""
    sc = Scene("gqa8x2d128", [900, 100], seed=14)
    n_q = [1, 70]
    q, out, lse = run(sc, n_q)
    run(sc, n_q, num_splits=4)  # the workspace exists before the capture
    o2, l2 = torch.zeros_like(out), torch.zeros_like(lse)
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        with torch.cuda.graph(graph, stream=st):
            sc.pool.extend(sc.ids, n_q, q, o2, l2)
    for _ in range(3):
        o2.zero_()
        l2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o2, out) and torch.equal(l2, lse)
        _, o3, l3 = run(sc, n_q, q=q)
        assert torch.equal(o3, out) and torch.equal(l3, lse)
    sc.close()
