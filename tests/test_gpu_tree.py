"""Attention of drafted trees over the pool (cp_tree_build, cp_attn_tree,
cp_attn_tree_step) against the 64-bit form: geometries, tree and page sizes,
masks, rows that see nothing, special values out of sight, ranges joined, shared
pages, rotated rows, layers, graphs."""
import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, Scene, bits, check, rounds_to_16_bits, shape, turn_rows
from token_ref import ancestors, attend_tree, make_tree, pack

pytestmark = pytest.mark.gpu


def device_tree(parents, words=None):
    """(mask, depth) on the GPU of trees given by their parents."""
    total = sum(len(p) for p in parents)
    words = words or max(1, -(-max(len(p) for p in parents) // 32))
    par = torch.tensor([x for p in parents for x in p], dtype=torch.int32, device="cuda")
    mask = torch.full((total, words), -1, dtype=torch.int32, device="cuda")
    depth = torch.full((total,), -5, dtype=torch.int32, device="cuda")
    cpl.cp_tree_build([len(p) for p in parents], par, mask, depth)
    return mask, depth


def verify(sc, parents, label, together=False, rows=None, sees=None, **opts):
    """The last tokens of every request are its tree; sees: masks of another kind."""
    n_q = [len(p) for p in parents]
    total = sum(n_q)
    q, out, lse = sc.buffers(total)
    if sees is None:
        mask, depth = device_tree(parents)
    else:
        words = -(-max(n_q) // 32)
        mask = torch.cat([pack(s, words) for s in sees]).cuda()
        depth = torch.cat([ancestors(p)[1] for p in parents]).cuda()
    sc.pool.tree(sc.ids, n_q, q, out, lse, mask, depth, **opts)
    torch.cuda.synchronize()
    path = opts.pop("path", cpl.CP_PATH_AUTO)
    opts.pop("num_splits", None)
    docs = opts.pop("doc_begin", None)
    at = 0
    for i, p in enumerate(parents):
        k = len(p)
        if k == 0:
            continue
        own, d = ancestors(p)
        ref = attend_tree(sc.name, (rows or sc.rows)[i], q[at:at + k], own if sees is None else sees[i], d,
                          doc_begin=docs[at:at + k] if docs is not None else None, **opts)
        check(out[at:at + k], lse[at:at + k], ref, together or rounds_to_16_bits(sc.name, k, path), f"{label} request {i}")
        at += k
    return q, out, lse, mask, depth


@pytest.mark.parametrize("n,words", [(1, 1), (31, 1), (32, 1), (33, 2), (64, 7), (300, 10), (4096, 128)])
def test_masks_and_depths(n, words):
    """Trees next to each other, chains, every parent a root, parents that are none."""
    for seed, kw in ((1, {}), (2, dict(width=1, roots=0.0)), (3, dict(roots=1.0)), (4, dict(width=n, roots=0.02))):
        trees = [make_tree(n, seed, **kw), make_tree(max(1, n // 3), seed + 10), make_tree(n, seed + 20)]
        if n > 3:
            trees[0][n // 2] = n // 2  # itself
            trees[0][n - 1] = n + 5    # none
            trees[0][1] = -2 ** 31
        if n > 1000:
            trees = trees[:1]
        mask, depth = device_tree(trees, words)
        want = [ancestors(t) for t in trees]
        assert torch.equal(depth.cpu(), torch.cat([d for _, d in want]))
        assert torch.equal(mask.cpu(), torch.cat([pack(s, words) for s, _ in want]))


def test_many_trees_take_several_launches():
    trees = [make_tree(1 + i % 40, i) for i in range(150)]
    mask, depth = device_tree(trees)
    want = [ancestors(t) for t in trees]
    assert torch.equal(depth.cpu(), torch.cat([d for _, d in want]))
    assert torch.equal(mask.cpu(), torch.cat([pack(s, 2) for s, _ in want]))


@pytest.mark.parametrize("name", sorted(GEOMS))
@pytest.mark.parametrize("path", [cpl.CP_PATH_AUTO, cpl.CP_PATH_VALU])
def test_trees_of_every_geometry(name, path):
    """One token, few, past a tile, the whole context."""
    print(f"[case] tree {name} path {path}", flush=True)
    sc = Scene(name, [1, 63, 200, 70], seed=3)
    verify(sc, [make_tree(1, 1), make_tree(5, 2), make_tree(70, 3), make_tree(70, 4)], f"{name} path {path}", path=path)
    verify(sc, [[], make_tree(2, 5), [], make_tree(1, 6)], f"{name} few path {path}", path=path)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("page_tokens", [1, 6, 16, 48, 150])
def test_page_sizes(name, page_tokens):
    if page_tokens * 2 * shape(name)[4] % 256:
        pytest.skip("pages of this model are no multiple of 256 bytes")
    print(f"[case] tree pages {name} {page_tokens}", flush=True)
    sc = Scene(name, [77, 210], page_tokens=page_tokens, seed=4)
    verify(sc, [make_tree(9, 1), make_tree(45, 2)], f"{name} P{page_tokens}")
    sc.close()


MASKS = {
    "cap": dict(softcap=3.0),
    "slopes": dict(slopes=True),
    "window": dict(window=37),
    "window 1": dict(window=1),
    "docs": dict(docs=True),
    "all": dict(softcap=5.0, slopes=True, window=90, docs=True),
}


@pytest.mark.parametrize("mask", sorted(MASKS))
@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mqa32d128", "mla20", "mla4l128r40"])
@pytest.mark.parametrize("n_q", [[1, 1, 1], [4, 2, 5], [8, 7, 6], [61, 40, 33]])
def test_masks(mask, name, n_q):
    print(f"[case] tree mask {mask} {name} {n_q}", flush=True)
    lens = [201, 130, 67]
    sc = Scene(name, lens, seed=5)
    opts = dict(MASKS[mask])
    if opts.pop("slopes", None):
        opts["slopes"] = torch.linspace(0.5, 0.01, sc.hq, device="cuda")
    if opts.pop("docs", None):  # some start inside the tree: the context is not seen, the tree is
        opts["doc_begin"] = torch.tensor([(41 * i) % n for n, k in zip(lens, n_q) for i in range(k)], dtype=torch.int32,
                                         device="cuda")
    verify(sc, [make_tree(k, 7 + k) for k in n_q], f"{mask} {name}", **opts)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l64r0"])
@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("splits", [0, 3])
def test_other_masks_and_rows_that_see_nothing(name, n, splits):
    """Masks that are no tree's: none, all, later tokens, and bits past the tree."""
    print(f"[case] tree other {name} {n} {splits}", flush=True)
    for ctx in (n, n + 150):  # (n: an empty mask leaves an empty row)
        sc = Scene(name, [ctx], seed=6)
        gen = torch.Generator().manual_seed(n)
        sees = torch.rand(n, 32 * -(-n // 32), generator=gen) < 0.5  # (bits past the tree among them)
        sees[0] = False
        sees[n // 2] = True
        verify(sc, [make_tree(n, 9)], f"{name} ctx {ctx}", sees=[sees], num_splits=splits)
        sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mqa32d128", "mla16", "mla128", "gqa4x2d256"])
@pytest.mark.parametrize("splits", [2, 5, 64])
@pytest.mark.parametrize("n", [1, 33])
def test_ranges_are_joined(name, splits, n):
    print(f"[case] tree splits {name} {splits} {n}", flush=True)
    sc = Scene(name, [900, 65], seed=7)
    trees = [make_tree(n, 3), make_tree(n, 4)]
    verify(sc, trees, f"{name} splits {splits}", num_splits=splits)
    verify(sc, trees, f"{name} splits {splits} window", num_splits=splits, window=100)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mqa32d128", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("n", [4, 40])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_special_values_out_of_sight_stay_there(name, n, bad):
    """A drafted token's K and V are special: the branches without it are not
    touched. One special element of V reaches those that see it, in its column."""
    print(f"[case] tree special {name} {n} {bad}", flush=True)
    ctx = 150
    hq, hkv, dk, dv, row, _ = shape(name)
    parents = [-1, -1, 0, 1] + [t - 2 for t in range(4, n)]  # two chains
    sees, depth = ancestors(parents)
    sc = Scene(name, [ctx], seed=8, fill=float("nan"))
    rows = sc.rows[0].clone()
    rows[ctx - n + 1, :] = bad  # the second chain's root
    sc.pool.truncate([sc.ids[0]], [0])
    sc.pool.append([sc.ids[0]], [ctx], rows)
    q, out, lse = sc.buffers(n)
    mask, d = device_tree([parents])
    sc.pool.tree(sc.ids, [n], q, out, lse, mask, d)
    torch.cuda.synchronize()
    clean = rows.clone()
    clean[ctx - n + 1] = 0
    ref = attend_tree(name, clean, q, sees, depth)
    first = ~sees[:, 1]
    check(out[first.cuda()], lse[first.cuda()], [x[first] for x in ref], rounds_to_16_bits(name, n), f"{name} {bad}")
    if GEOMS[name]["kind"] == cpl.CP_KIND_GQA and bad == bad:
        rows = sc.rows[0].clone()
        rows[ctx - n + 1, hkv * dk + 5] = bad
        sc.pool.truncate([sc.ids[0]], [0])
        sc.pool.append([sc.ids[0]], [ctx], rows)
        sc.pool.tree(sc.ids, [n], q, out, lse, mask, d)
        torch.cuda.synchronize()
        got = out.float().cpu()
        g = hq // hkv
        assert torch.equal(got[~first][:, :g, 5], torch.full((int((~first).sum()), g), bad))
        assert torch.isfinite(got[first]).all()
        got[:, :g, 5] = 0
        assert torch.isfinite(got).all()
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16"])
@pytest.mark.parametrize("slopes", [False, True])
def test_a_chain_is_a_chunk(name, slopes):
    """A tree that is one chain: the same as cp_attn_extend of its tokens."""
    sc = Scene(name, [500, 80], seed=10)
    opts = dict(slopes=torch.linspace(0.3, 0.01, sc.hq, device="cuda")) if slopes else {}
    trees = [list(range(-1, 39)), list(range(-1, 4))]
    q, out, lse, _, _ = verify(sc, trees, name, window=60, **opts)
    o2, l2 = torch.zeros_like(out), torch.zeros_like(lse)
    sc.pool.extend(sc.ids, [40, 5], q, o2, l2, window=60, **opts)
    torch.cuda.synchronize()
    assert torch.allclose(lse, l2, atol=1e-4)
    # each off by half a step of the output, and of probabilities times |v| (under 0.7 * 6)
    assert ((out.float() - o2.float()).abs() <= 2.0 ** -7 * out.float().abs() + 2.0 ** -7 * 0.7 * 6).all()
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mqa32d128", "mla16"])
@pytest.mark.parametrize("mask", ["none", "all"])
@pytest.mark.parametrize("sizes", [[1, 3, 5, 2], [20, 9, 31, 17]])
def test_forks_read_their_shared_pages_once(name, mask, sizes):
    """Branches of one prompt, each with a tree of its own; the last one's tree lies in
    pages that another request shows too."""
    print(f"[case] tree shared {name} {mask} {sizes}", flush=True)
    shared = 1000
    sc = Scene(name, [shared], seed=15, room=100, pool_bytes=256 << 20)
    kids, rows = [], []
    for k in sizes:
        rid = sc.pool.open(sc.model, shared + 400)
        sc.pool.fork([sc.ids[0]], [rid])
        tail = sc.normal(k, sc.row, sigma=0.7)
        sc.pool.append([rid], [k], tail)
        kids.append(rid)
        rows.append(torch.cat([sc.rows[0], tail]))
    sc.ids, sc.rows = kids + sc.ids, rows + sc.rows
    opts = {}
    if mask == "all":
        opts = dict(softcap=8.0, window=700, slopes=torch.linspace(0.3, 0.01, sc.hq, device="cuda"))
    verify(sc, [make_tree(k, k) for k in sizes] + [make_tree(sizes[-1], 3)], f"{name} {mask}", together=True, **opts)
    sc.close()


@pytest.mark.parametrize("name,layout,rot", [("gqa8x2d128", "half", 64), ("gqa6x2d64", "interleaved", 64),
                                             ("mla16", "interleaved", 64), ("mla4l128r40", "half", 40)])
def test_steps_place_rows_turned_by_depth(name, layout, rot):
    """Two layers, trees of several sizes over page ends: rows gathered, outputs, cursors."""
    print(f"[case] tree step {name}", flush=True)
    lens = [62, 130, 0]
    sizes = [5, 70, 33]
    sc = Scene(name, lens, seed=11, room=100, layers=2)
    rope = cpl.Rope(rot, layout=layout)
    trees = [make_tree(k, k + 1) for k in sizes]
    own = [ancestors(t) for t in trees]
    mask, depth = device_tree(trees)
    total = sum(sizes)
    held = [r.clone() if r.dim() == 3 else r for r in sc.rows]
    for layer in range(2):
        new = sc.normal(total, sc.row, sigma=0.7)
        q, out, lse = sc.buffers(total)
        sc.pool.tree_step(sc.ids, sizes, new, q, out, lse, mask, depth, rope=rope)
        torch.cuda.synchronize()
        at = 0
        for i, k in enumerate(sizes):
            pos = lens[i] + own[i][1].long()
            assert sc.pool.cursor(sc.ids[i]) == ((1, k) if layer == 0 else (0, 0))
            if layer == 1:
                got = sc.held(sc.ids[i], lens[i] + k, layers=2)
                assert torch.equal(got[:, :lens[i]], held[i])
                g = got[1, lens[i]:].double().cpu()
                w64 = turn_rows(name, new[at:at + k], rope.angles(), pos, layout)
                # one rounding to bf16 (half a step of the value) of sums in 32 bits, 2^-20 of the pair
                assert ((g - w64).abs() <= 2.0 ** -8 * w64.abs() + 2.0 ** -18).all()
                ref = attend_tree(name, got[1], q[at:at + k], *own[i])
                check(out[at:at + k], lse[at:at + k], ref, rounds_to_16_bits(name, k), f"{name} layer {layer} request {i}")
            at += k
    rope.destroy()
    sc.close()


def test_steps_of_requests_without_a_tree():
    """Their cursors move on, and the others' trees are as alone."""
    print("[case] tree step, some without", flush=True)
    lens, sizes = [20, 64, 33], [0, 6, 0]
    held = []
    mask, depth = device_tree([make_tree(6, 2)])
    for some in ([0, 1, 2], [1]):
        sc = Scene("gqa8x2d128", lens, seed=13, room=20, layers=2)
        for layer in range(2):
            sc.gen.manual_seed(50 + layer)
            new = sc.normal(6, sc.row, sigma=0.7)
            q, out, lse = sc.buffers(6)
            sc.pool.tree_step([sc.ids[i] for i in some], [sizes[i] for i in some], new, q, out, lse, mask, depth)
            held.append((out, lse))
            want = (1, 0) if layer == 0 else (0, 0)
            assert all(sc.pool.cursor(sc.ids[i]) == want for i in some if i != 1)
        assert [sc.pool.ctx_len(i) for i in sc.ids] == [20, 70, 33]
        held.append((sc.held(sc.ids[1], 70, layers=2),) * 2)
        torch.cuda.synchronize()
        sc.close()
    for x, y in zip(held[:3], held[3:]):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_depths_out_of_range_count_as_the_last():
    """Positions of queries and of rotated keys, and distances of keys, alike."""
    print("[case] depths out of range", flush=True)
    n, k = 90, 7
    rope = cpl.Rope(64, layout="half")
    slopes = torch.linspace(0.5, 0.01, 16, device="cuda")
    mask, depth = device_tree([[-1, 0, 0, 1, 1, 2, 2]])
    for at, bad in ((3, -1), (5, 1000), (0, -(2 ** 31)), (6, 2 ** 31 - 1)):
        held = []
        for value in (bad, k - 1):
            sc = Scene("gqa8x2d128", [n], seed=12, room=20)
            new = sc.normal(k, sc.row, sigma=0.7)
            q, out, lse = sc.buffers(k)
            d = depth.clone()
            d[at] = value
            sc.pool.tree_step(sc.ids, [k], new, q, out, lse, mask, d, rope=rope, slopes=slopes[:sc.hq])
            held.append((out, lse, sc.held(sc.ids[0], n + k)))
            torch.cuda.synchronize()
            sc.close()
        for x, y in zip(*held):
            assert torch.equal(x, y)
    rope.destroy()


def test_many_requests_take_several_launches():
    lens = [40 + (37 * i) % 90 for i in range(100)]
    sc = Scene("gqa6x2d64", lens, seed=12)
    verify(sc, [make_tree(1 + i % 12, i) for i in range(100)], "100 requests")
    sc.close()


def test_long_context():
    """A wide tree over 70,001 tokens, planned ranges, slopes and a cap."""
    sc = Scene("gqa8x2d128", [70001], seed=13)
    verify(sc, [make_tree(40, 1)], "long", slopes=torch.linspace(0.01, 1e-5, 8, device="cuda"), softcap=30.0)
    sc.close()


def test_graph_replays_and_streams():
    """Masks and attention captured together, parents changed between replays."""
    sc = Scene("gqa8x2d128", [900, 100], seed=14)
    sizes = [7, 30]
    first, second = [make_tree(k, 1) for k in sizes], [make_tree(k, 2) for k in sizes]
    q, out, lse = sc.buffers(37)
    mask, depth = device_tree(first)
    sc.pool.tree(sc.ids, sizes, q, out, lse, mask, depth)  # the workspace exists before the capture
    par = torch.tensor(sum(first, []), dtype=torch.int32, device="cuda")
    o2, l2 = torch.zeros_like(out), torch.zeros_like(lse)
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        with torch.cuda.graph(graph, stream=st):
            cpl.cp_tree_build(sizes, par, mask, depth)
            sc.pool.tree(sc.ids, sizes, q, o2, l2, mask, depth)
    for trees in (second, first, second):
        par.copy_(torch.tensor(sum(trees, []), dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        m, d = device_tree(trees)
        sc.pool.tree(sc.ids, sizes, q, out, lse, m, d)
        torch.cuda.synchronize()
        assert torch.equal(o2, out) and torch.equal(l2, lse)
    sc.close()
