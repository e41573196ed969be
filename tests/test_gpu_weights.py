"""Weights that queries give to cached tokens (cp_attn_weights) against the 64-bit
form: geometries, lengths, masks, rows that saw nothing, sums that decay, strides,
special values, parts joined, layers, graphs, streams."""
import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, Scene, attend, shape
from token_ref import given

pytestmark = pytest.mark.gpu


def compare(got, want_new, old, decay, label):
    """Allowed: 2^-11 of the new weights (scores of up to 2^6 off by at most 2^-12, as in
    the attention's tests, lse times log2 e off by 2^-24 of at most 2^7, the exponential and
    sums of up to 2^11 rows 2^-13: together below 2^-11), 2^-22 of the whole (the decayed
    sum and the last addition round once each), and what is too small for 32 bits."""
    total = want_new + (old.double().cpu() * decay if old is not None and decay else 0.0)
    tol = 2.0 ** -11 * want_new + 2.0 ** -22 * total + 1e-30
    err = (got.double().cpu() - total).abs()
    worst = (err / tol).max().item()
    print(f"[weights] {label} {worst:.3f} of the tolerance", flush=True)
    assert torch.isfinite(got).all(), label
    assert worst <= 1, (label, worst)


def scene_queries(sc, n_q, rows=None, **opts):
    """Queries of the last tokens, and their log-sum-exp by the 64-bit form, in 32 bits."""
    total = sum(n_q)
    q = sc.normal(total, sc.hq, sc.dk)
    lse = torch.zeros(total, sc.hq)
    prefix, docs = opts.pop("prefix", None), opts.pop("doc_begin", None)
    at = 0
    for i, k in enumerate(n_q):
        if k:
            lse[at:at + k] = attend(sc.name, (rows or sc.rows)[i], q[at:at + k], prefix=prefix[i] if prefix else 0,
                                    doc_begin=docs[at:at + k] if docs is not None else None, **opts)[1].float()
        at += k
    return q, lse.cuda()


def verify(sc, n_q, label, decay=0.0, pad=0, path=cpl.CP_PATH_AUTO, num_splits=0, **opts):
    q, lse = scene_queries(sc, n_q, **opts)
    lens = [r.shape[0] for r in sc.rows]
    room = [torch.rand(sc.hkv, n + pad, device="cuda") for n in lens]
    new = [torch.full((sc.hkv, n + pad), 7.0, device="cuda") for n in lens]
    old = [r[:, :n] for r, n in zip(room, lens)] if decay else None
    sc.pool.weights(sc.ids, n_q, q, lse, new, old=old, decay=decay, path=path, num_splits=num_splits, **opts)
    torch.cuda.synchronize()
    prefix, docs = opts.pop("prefix", None), opts.pop("doc_begin", None)
    at = 0
    for i, k in enumerate(n_q):
        n = lens[i]
        want = given(sc.name, sc.rows[i], q[at:at + k], lse[at:at + k], prefix=prefix[i] if prefix else 0,
                     doc_begin=docs[at:at + k] if docs is not None else None, **opts)
        compare(new[i][:, :n], want, old[i] if old else None, decay, f"{label} request {i}")
        assert (new[i][:, n:] == 7.0).all()
        at += k
    return q, lse, new


@pytest.mark.parametrize("name", sorted(GEOMS))
@pytest.mark.parametrize("path", [cpl.CP_PATH_AUTO, cpl.CP_PATH_VALU])
def test_every_geometry(name, path):
    """One token, a few, blocks and tiles that end anywhere, and none."""
    print(f"[case] weights {name} path {path}", flush=True)
    sc = Scene(name, [1, 63, 200, 129, 530], seed=3)
    verify(sc, [1, 1, 7, 129, 70], f"{name} path {path}", path=path)
    verify(sc, [0, 3, 0, 1, 2], f"{name} decay path {path}", path=path, decay=0.75, pad=5)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("page_tokens", [1, 6, 16, 48, 150])
def test_page_sizes(name, page_tokens):
    if page_tokens * 2 * shape(name)[4] % 256:
        pytest.skip("pages of this model are no multiple of 256 bytes")
    print(f"[case] weights pages {name} {page_tokens}", flush=True)
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
    print(f"[case] weights mask {mask} {name} {n_q}", flush=True)
    lens = [301, 130, 67]
    sc = Scene(name, lens, seed=5)
    opts = dict(MASKS[mask])
    if opts.pop("slopes", None):
        opts["slopes"] = torch.linspace(0.5, 0.01, sc.hq, device="cuda")
    if opts.pop("docs", None):
        starts = []
        for n, k in zip(lens, n_q):
            starts += [max(0, (p // 23) * 23 - 5) for p in range(n - k, n)]
        opts["doc_begin"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    verify(sc, n_q, f"{mask} {name}", decay=1.0, **opts)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l64r0"])
@pytest.mark.parametrize("n_q", [2, 90])
def test_rows_that_saw_nothing_give_nothing(name, n_q):
    """Documents behind a token: no key is seen, lse is -inf; all of them, and some."""
    print(f"[case] weights empty {name} {n_q}", flush=True)
    sc = Scene(name, [300], seed=6)
    some = torch.tensor([300 if i % 3 == 0 else -7 for i in range(n_q)], dtype=torch.int32, device="cuda")
    verify(sc, [n_q], f"{name} some", doc_begin=some)
    none = torch.full((n_q,), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
    _, lse, new = verify(sc, [n_q], f"{name} none", doc_begin=none)
    assert torch.isinf(lse).all() and (new[0] == 0).all()
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("splits", [2, 5, 64])
def test_parts_are_joined(name, splits):
    print(f"[case] weights splits {name} {splits}", flush=True)
    sc = Scene(name, [600, 65], seed=7)
    verify(sc, [300, 65], f"{name} splits {splits}", num_splits=splits, decay=0.5)
    verify(sc, [300, 65], f"{name} splits {splits} window", num_splits=splits, window=100)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "gqa6x2d64", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("n_q", [3, 70])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_special_keys_stay_where_they_are(name, n_q, bad):
    """A key that some rows do not see, stale memory behind the context, and a row whose
    own log-sum-exp is NaN: only what they touch is touched."""
    print(f"[case] weights special {name} {n_q} {bad}", flush=True)
    n = 210
    hq, hkv = shape(name)[:2]
    sc = Scene(name, [n], seed=8, fill=float("nan"))
    q, lse = scene_queries(sc, [n_q])
    where = n - 2
    sc.pool.truncate([sc.ids[0]], [where])
    rows = sc.rows[0].clone()
    rows[where] = bad
    sc.pool.append([sc.ids[0]], [n - where], rows[where:].contiguous())
    new = [torch.zeros(hkv, n, device="cuda")]
    sc.pool.weights(sc.ids, [n_q], q, lse, new)
    torch.cuda.synchronize()
    want = given(name, sc.rows[0], q, lse)
    rest = [j for j in range(n) if j != where]
    compare(new[0][:, rest], want[:, rest], None, 0, f"{name} {bad}")
    # a NaN row: the keys it sees, of its KV head
    sc.pool.truncate([sc.ids[0]], [where])
    sc.pool.append([sc.ids[0]], [n - where], sc.rows[0][where:].contiguous())
    lse[0, 0] = float("nan")
    sc.pool.weights(sc.ids, [n_q], q, lse, new, window=50)
    torch.cuda.synchronize()
    got = new[0].cpu()
    p = n - n_q
    sees = torch.zeros(n, dtype=torch.bool)
    sees[max(0, p - 49):p + 1] = True
    assert torch.equal(torch.isnan(got[0]), sees) and torch.isfinite(got[1:]).all()
    sc.close()


def test_sums_go_on_in_place_and_by_strides():
    """old and new the same memory; rows of heads and layers far apart."""
    sc = Scene("gqa8x2d128", [90, 500], seed=9, layers=1)
    q, lse = scene_queries(sc, [1, 40])
    big = torch.rand(2, 3, 700, device="cuda")  # [request][.][tokens]: a KV head in rows 0 and 2
    keep = big.clone()
    views = [big[0, ::2, :90], big[1, ::2, :500]]
    olds = [v.clone() for v in views]
    sc.pool.weights(sc.ids, [1, 40], q, lse, views, old=views, decay=0.9)
    torch.cuda.synchronize()
    for i, (k, at) in enumerate(((1, 0), (40, 1))):
        compare(views[i], given(sc.name, sc.rows[i], q[at:at + k], lse[at:at + k]), olds[i], 0.9, f"request {i}")
    assert torch.equal(big[:, 1], keep[:, 1]) and torch.equal(big[0, :, 90:], keep[0, :, 90:])
    assert torch.equal(big[1, :, 500:], keep[1, :, 500:])
    sc.close()


def test_layers_and_tokens_in_flight():
    """Each layer's keys, and its own rows of the sums; a token in flight counts in the
    layers that its steps have passed."""
    sc = Scene("gqa8x2d128", [130], seed=10, layers=3, room=10)
    rows = sc.rows[0]
    w = [torch.zeros(3, 2, 140, device="cuda")]
    extra = sc.normal(5, sc.row, sigma=0.7)
    q5, out, l5 = sc.buffers(5)
    sc.pool.extend_step(sc.ids, [5], extra, q5, out, l5)  # layer 0 passed
    for layer, n in ((0, 135), (1, 130), (2, 130)):
        held = torch.cat([rows[layer], extra]) if layer == 0 else rows[layer]
        q = sc.normal(33, sc.hq, sc.dk)
        lse = attend(sc.name, held, q)[1].float().cuda()
        sc.pool.weights(sc.ids, [33], q, lse, w, layer=layer)
        torch.cuda.synchronize()
        compare(w[0][layer, :, :n], given(sc.name, held, q, lse), None, 0, f"layer {layer}")
        assert (w[0][layer, :, n:] == 0).all() and (w[0][layer + 1:] == 0).all()
    for _ in range(2):
        sc.pool.extend_step(sc.ids, [5], extra, q5, out, l5)
    sc.close()


def test_weights_of_a_softmax_add_up():
    """With the lse of this library's own attention each row gives 1 in all."""
    for name in ("gqa8x2d128", "mla16", "gqa6x2d64", "mla4l128r40"):
        sc = Scene(name, [1000, 333], seed=11)
        n_q = [100, 1]
        q, out, lse = sc.buffers(101)
        sc.pool.extend(sc.ids, n_q, q, out, lse)
        new = [torch.zeros(sc.hkv, n, device="cuda") for n in (1000, 333)]
        sc.pool.weights(sc.ids, n_q, q, lse, new)
        torch.cuda.synchronize()
        g = sc.hq // sc.hkv
        for w, k in zip(new, n_q):
            # each score and lse off by at most 2^-12 of their own
            assert (w.double().sum(1).cpu() - k * g).abs().max() <= 2.0 ** -10 * k * g
        sc.close()


def test_many_requests_and_long_contexts():
    lens = [1 + (37 * i) % 190 for i in range(90)]
    sc = Scene("gqa6x2d64", lens, seed=12)
    verify(sc, [min(n, 1 + i % 12) for i, n in enumerate(lens)], "90 requests", decay=0.5)
    sc.close()
    sc = Scene("gqa8x2d128", [70001], seed=13)
    verify(sc, [1], "long", slopes=torch.linspace(0.01, 1e-5, 8, device="cuda"), softcap=30.0)
    verify(sc, [65], "long window", window=65536)
    sc.close()


def test_results_do_not_depend_on_placement_or_company():
    sc = Scene("gqa8x2d128", [700, 300, 50], seed=14)
    n_q = [65, 3, 1]
    q, lse = scene_queries(sc, n_q)
    new = [torch.zeros(2, n, device="cuda") for n in (700, 300, 50)]
    sc.pool.weights(sc.ids, n_q, q, lse, new, num_splits=3)
    other = Scene("gqa8x2d128", [700], seed=99)
    other.pool.truncate(other.ids, [0])
    other.pool.append(other.ids, [700], sc.rows[0])
    w = [torch.zeros(2, 700, device="cuda")]
    other.pool.weights(other.ids, [65], q[:65].contiguous(), lse[:65].contiguous(), w, num_splits=3)
    torch.cuda.synchronize()
    assert torch.equal(w[0], new[0])
    other.close()
    sc.close()


def test_graph_replays_and_streams():
    """Captured and replayed, the sums growing from replay to replay, eager calls between."""
    sc = Scene("gqa8x2d128", [900, 100], seed=15)
    n_q = [200, 1]
    q, lse = scene_queries(sc, n_q)
    a = [torch.zeros(2, n, device="cuda") for n in (900, 100)]
    b = [torch.zeros(2, n, device="cuda") for n in (900, 100)]
    sc.pool.weights(sc.ids, n_q, q, lse, a, num_splits=3)  # the workspace exists before the capture
    for w in a:
        w.zero_()
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        with torch.cuda.graph(graph, stream=st):
            sc.pool.weights(sc.ids, n_q, q, lse, b, old=b, decay=0.5, num_splits=3)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        sc.pool.weights(sc.ids, n_q, q, lse, a, old=a, decay=0.5, num_splits=3)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    sc.close()
