"""Keeping some of a request's tokens: accepted paths (cp_request_keep) and evictions by
weight (cp_kv_evict) against rows picked on the host, bit for bit: geometries, page
sizes, layers, shared pages, ties and special weights, places of the rows' memory, both
backings, device page stacks, positions of what comes next."""
import random

import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, Scene, check, rounds_to_16_bits, shape, turn_rows
from token_ref import ancestors, attend_tree, given, heaviest, kept_rows, make_tree, pack

pytestmark = pytest.mark.gpu


def pick(n, k, seed):
    return sorted(random.Random(seed).sample(range(n), k))


@pytest.mark.parametrize("name", sorted(GEOMS))
@pytest.mark.parametrize("layers", [1, 3])
def test_kept_tokens_of_every_geometry(name, layers):
    """Lists of all kinds, several requests in a call; what comes behind is gone."""
    print(f"[case] keep {name} {layers}", flush=True)
    lens = [1, 70, 300, 64, 200]
    sc = Scene(name, lens, seed=3, layers=layers, room=20)
    rows = [r if r.dim() == 3 else r[None] for r in sc.rows]
    first = [0, 60, 100, 64, 0]
    lists = [[0], pick(10, 4, 1), pick(200, 90, 2), [], [3, 4, 5, 199]]
    sc.pool.keep(sc.ids, first, [len(x) for x in lists], sum(lists, []))
    for i, (f, l) in enumerate(zip(first, lists)):
        want = torch.cat([rows[i][:, :f], rows[i][:, f:][:, l]], dim=1)
        assert sc.pool.ctx_len(sc.ids[i]) == f + len(l) == sc.pool.position(sc.ids[i])
        assert torch.equal(sc.held(sc.ids[i], f + len(l), layers).view(want.shape), want), i
    # and they go on
    new = sc.normal(layers, 9, sc.row)
    sc.pool.append([sc.ids[2]], [9], new)
    assert torch.equal(sc.held(sc.ids[2], 199, layers).view(layers, 199, -1)[:, 190:], new)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "mla16", "mla4l128r40"])
@pytest.mark.parametrize("page_tokens", [1, 6, 16, 150])
@pytest.mark.parametrize("n", [900])
def test_long_lists_and_page_sizes(name, page_tokens, n):
    """More than one launch carries, and steps of many rows in place."""
    if page_tokens * 2 * shape(name)[4] % 256:
        pytest.skip("pages of this model are no multiple of 256 bytes")
    print(f"[case] keep long {name} {page_tokens}", flush=True)
    sc = Scene(name, [n, n], page_tokens=page_tokens, seed=4)
    lists = [pick(n - 3, 700, 5), pick(n, 899, 6)]
    sc.pool.keep(sc.ids, [3, 0], [700, 899], lists[0] + lists[1])
    assert torch.equal(sc.held(sc.ids[0], 703), torch.cat([sc.rows[0][:3], sc.rows[0][3:][lists[0]]]))
    assert torch.equal(sc.held(sc.ids[1], 899), sc.rows[1][lists[1]])
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "mla16"])
@pytest.mark.parametrize("backing", ["buffer", "virtual", "device pages"])
def test_shared_pages_are_replaced(name, backing):
    """Forks whose pages rows would move into, in one call with their source."""
    print(f"[case] keep shared {name} {backing}", flush=True)
    kw = {"virtual": dict(backing=cpl.CP_BACKING_VIRTUAL), "device pages": dict(device_pages=1)}.get(backing, {})
    sc = Scene(name, [400], seed=5, room=200, pool_bytes=256 << 20, **kw)
    a, rows = sc.ids[0], sc.rows[0]
    b, c = sc.pool.open(sc.model, 600), sc.pool.open(sc.model, 600)
    sc.pool.fork([a, a], [b, c], [400, 320])
    lists = [pick(300, 80, 7), pick(390, 200, 8)]
    sc.pool.keep([a, b], [100, 10], [80, 200], lists[0] + lists[1])
    assert torch.equal(sc.held(a, 180), torch.cat([rows[:100], rows[100:][lists[0]]]))
    assert torch.equal(sc.held(b, 210), torch.cat([rows[:10], rows[10:][lists[1]]]))
    assert torch.equal(sc.held(c, 320), rows[:320])
    sc.pool.append([a, b, c], [30, 30, 30], torch.cat([sc.normal(30, sc.row)] * 3))
    assert torch.equal(sc.held(c, 320), rows[:320])
    assert torch.equal(sc.held(a, 100), rows[:100]) and torch.equal(sc.held(b, 10), rows[:10])
    # a prefix of the list is where it belongs: pages before the first move stay shared
    before = sc.pool.stats()["pages_used"]
    d = sc.pool.open(sc.model, 600)
    sc.pool.fork([c], [d])
    shared = sc.pool.stats()["pages_used"]
    sc.pool.keep([d], [0], [300], list(range(299)) + [310])
    assert sc.pool.stats()["pages_used"] == shared and before <= shared
    assert torch.equal(sc.held(d, 300), torch.cat([rows[:299], rows[310:311]]))
    sc.ids = [a, b, c, d]
    sc.close()
    # (a closed scene returns every page: its destroy would fail otherwise)


WEIGHTS = ["normal", "equal", "zeros", "steps", "special", "tiny", "negative"]


def weights_of(kind, layers, hkv, n, seed):
    gen = torch.Generator().manual_seed(seed)
    w = torch.randn(layers, hkv, n, generator=gen).mul(3).exp()
    if kind == "equal":
        w = torch.full_like(w, 0.25)
    elif kind == "zeros":
        w = w * (torch.rand(w.shape, generator=gen) < 0.1)
    elif kind == "steps":
        w = torch.randint(0, 4, w.shape, generator=gen).float()
    elif kind == "special":
        x = torch.tensor([float("nan"), float("inf"), float("-inf"), -0.0, 0.0, 1.0, 1.0])
        w = x[torch.randint(0, 7, w.shape, generator=gen)]
    elif kind == "tiny":
        w = torch.randint(0, 5, w.shape, generator=gen).float() * 2.0 ** -149 + (torch.rand(w.shape, generator=gen) < 0.5) * 1e38
    elif kind == "negative":
        w = -w
    return w


def evict(sc, ids, rows, keep, kind, first=0, last=0, seed=1, in_place=False, ask=True):
    """An eviction of these requests, checked."""
    layers = rows[0].shape[0]
    ws = [weights_of(kind, layers, sc.hkv, r.shape[1], seed + i) for i, r in enumerate(rows)]
    dev = [w.cuda() for w in ws]
    new = dev if in_place else [torch.full((layers, sc.hkv, w.shape[2] + 3), 7.0, device="cuda") for w in ws]
    kept = [torch.full((layers, sc.hkv, max(1, min(k, r.shape[1]))), -1, dtype=torch.int32, device="cuda")
            for k, r in zip(keep, rows)]
    at = [sc.pool.position(i) for i in ids]
    sc.pool.evict(ids, keep, dev, new=new, kept=kept if ask else None, first=first, last=last)
    torch.cuda.synchronize()
    out = []
    for i, rid in enumerate(ids):
        n, k = rows[i].shape[1], min(keep[i], rows[i].shape[1])
        want = [[heaviest(ws[i][l, h].tolist(), k, first, last) for h in range(sc.hkv)] for l in range(layers)]
        if ask and k:
            assert kept[i].cpu().tolist() == want, (kind, i)
        moved = kept_rows(sc.name, rows[i], want)
        assert sc.pool.ctx_len(rid) == k and sc.pool.position(rid) == at[i]
        assert torch.equal(sc.held(rid, k, layers).view(moved.shape).cpu().view(torch.int16), moved.view(torch.int16)), (kind, i)
        got = new[i].cpu()
        for l in range(layers):
            for h in range(sc.hkv):
                assert torch.equal(got[l, h, :k].view(torch.int32), ws[i][l, h][want[l][h]].view(torch.int32))
        assert (got[:, :, k:n] == 0).all() and (in_place or (got[:, :, n:] == 7).all())
        out.append(moved)
    return out


@pytest.mark.parametrize("name", sorted(GEOMS))
@pytest.mark.parametrize("layers", [1, 2])
def test_evictions_of_every_geometry(name, layers):
    """Lengths from one token on, everything, nothing, and no change."""
    print(f"[case] evict {name} {layers}", flush=True)
    lens = [1, 70, 300, 64, 200, 5]
    sc = Scene(name, lens, seed=3, layers=layers, room=20)
    rows = [r if r.dim() == 3 else r[None] for r in sc.rows]
    evict(sc, sc.ids, rows, [0, 30, 129, 64, 199, 100], "normal")
    sc.close()


@pytest.mark.parametrize("kind", WEIGHTS)
@pytest.mark.parametrize("n,keep,first,last", [(300, 100, 0, 0), (300, 100, 4, 96), (5000, 1200, 3, 50), (5000, 4999, 0, 0),
                                               (5000, 60, 60, 0), (1025, 1, 0, 0)])
def test_choices(kind, n, keep, first, last):
    print(f"[case] evict {kind} {n} {keep} {first} {last}", flush=True)
    sc = Scene("gqa8x2d128", [n, n - 7], seed=4)
    rows = [r[None] for r in sc.rows]
    evict(sc, sc.ids, rows, [keep, min(keep, n - 8)], kind, first, min(last, keep - first - 8) if last > 8 else last,
          in_place=kind in ("normal", "steps"), ask=kind != "zeros")
    sc.close()


def test_long_rows():
    """100,001 tokens: steps of many rows in place, and in pages of their own."""
    n = 100001
    sc = Scene("mla4l64r0", [n], seed=5, pool_bytes=64 << 20)
    b = sc.pool.open(sc.model, n)
    sc.pool.fork([sc.ids[0]], [b])
    rows = [sc.rows[0][None]]
    evict(sc, [b], rows, [33333], "normal", 10, 1000)
    evict(sc, sc.ids, rows, [70000], "zeros", 10, 1000)
    sc.ids.append(b)
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "mla16", "gqa6x2d64"])
@pytest.mark.parametrize("backing", ["buffer", "virtual", "device pages"])
@pytest.mark.parametrize("layers", [1, 12])
def test_evictions_of_shared_pages(name, backing, layers):
    """Branches and their prompt in one call and in calls of their own, entries that travel
    with the launch and (many) by a copy; the others keep what they had."""
    print(f"[case] evict shared {name} {backing} {layers}", flush=True)
    kw = {"virtual": dict(backing=cpl.CP_BACKING_VIRTUAL), "device pages": dict(device_pages=1)}.get(backing, {})
    n = 1500
    sc = Scene(name, [n], page_tokens=16, seed=5, layers=layers, room=200, pool_bytes=(64 << 20) * layers, **kw)
    a, rows = sc.ids[0], (sc.rows[0] if layers > 1 else sc.rows[0][None])
    b, c, d = (sc.pool.open(sc.model, n + 200) for _ in range(3))
    sc.pool.fork([a, a, a], [b, c, d], [n, n - 1, 800])
    evict(sc, [b], [rows], [500], "normal", 20, 30)
    evict(sc, [a, c], [rows, rows[:, :n - 1]], [700, 1490], "steps", 33, 30)
    assert torch.equal(sc.held(d, 800, layers).view(layers, 800, -1), rows[:, :800])
    tail = sc.normal(layers, 40, sc.row)
    for r, k in ((a, 700), (b, 500), (c, 1490), (d, 800)):
        sc.pool.append([r], [40], tail)
        assert torch.equal(sc.held(r, k + 40, layers).view(layers, k + 40, -1)[:, k:], tail)
    sc.pool.close(a)
    left = sc.held(b, 540, layers).view(layers, 540, -1)
    evict(sc, [b], [left], [100], "normal", 0, 0, seed=9)
    sc.ids = [b, c, d]
    sc.close()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_what_comes_next_stands_behind_what_was(layout):
    """Keys appended after an eviction are turned by the position they would have had."""
    sc = Scene("gqa8x2d128", [200], seed=6, room=40)
    rope = cpl.Rope(128, layout=layout)
    rid = sc.ids[0]
    evict(sc, [rid], [sc.rows[0][None]], [50], "normal")
    assert sc.pool.position(rid) == 200
    new = sc.normal(20, sc.row)
    sc.pool.append_rope([rid], [20], new, rope)
    want = turn_rows(sc.name, new, rope.angles(), torch.arange(200, 220), layout)
    got = sc.held(rid, 70)[50:].double().cpu()
    # one rounding to bf16 of sums in 32 bits
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18).all()
    branch = sc.pool.open(sc.model, 100)
    sc.pool.fork([rid], [branch], [60])
    assert sc.pool.position(branch) == 210
    q, out, lse = sc.buffers(5)
    sc.pool.extend_step([branch], [5], new[:5].contiguous(), q, out, lse, rope=rope)
    want = turn_rows(sc.name, new[:5], rope.angles(), torch.arange(210, 215), layout)
    got = sc.held(branch, 65)[60:].double().cpu()
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18).all()
    sc.pool.truncate([branch], [0])
    assert sc.pool.position(branch) == 0
    sc.ids.append(branch)
    rope.destroy()
    sc.close()


@pytest.mark.parametrize("name,rot", [("gqa8x2d128", 128), ("mla16", 64)])
def test_a_run_of_them_together(name, rot):
    """A decode with drafted trees: place, attend, keep the accepted path, weigh, and when
    the cache is full evict; against the rows and attention of the same steps on the host."""
    print(f"[case] run {name}", flush=True)
    rng = random.Random(1)
    budget, held = 260, [180, 250]
    sc = Scene(name, held, seed=7, room=400)
    rope = cpl.Rope(rot)
    rows = [r.clone() for r in sc.rows]
    sums = [torch.zeros(sc.hkv, 700, device="cuda") for _ in held]
    positions = list(held)
    for step in range(6):
        trees = [make_tree(rng.randint(3, 40), rng.random()) for _ in held]
        sizes = [len(t) for t in trees]
        own = [ancestors(t) for t in trees]
        total = sum(sizes)
        par = torch.tensor(sum(trees, []), dtype=torch.int32, device="cuda")
        mask = torch.zeros(total, 2, dtype=torch.int32, device="cuda")
        depth = torch.zeros(total, dtype=torch.int32, device="cuda")
        new = sc.normal(total, sc.row, sigma=0.7)
        q, out, lse = sc.buffers(total)
        cpl.cp_tree_build(sizes, par, mask, depth)
        sc.pool.tree_step(sc.ids, sizes, new, q, out, lse, mask, depth, rope=rope)
        paths = []
        for t in trees:
            node, path = rng.randrange(len(t)), []
            while node >= 0:
                path.append(node)
                node = t[node]
            paths.append(path[::-1])
        at = 0
        for i, k in enumerate(sizes):
            got = sc.held(sc.ids[i], rows[i].shape[0] + k)
            assert torch.equal(got[:rows[i].shape[0]], rows[i])
            want = turn_rows(name, new[at:at + k], rope.angles(), positions[i] + own[i][1].long(), "half")
            assert ((got[rows[i].shape[0]:].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18).all()
            ref = attend_tree(name, got, q[at:at + k], *own[i])
            check(out[at:at + k], lse[at:at + k], ref, rounds_to_16_bits(name, k), f"step {step} request {i}")
            rows[i] = torch.cat([rows[i], got[rows[i].shape[0]:][paths[i]]])
            at += k
        first = [sc.pool.ctx_len(r) - k for r, k in zip(sc.ids, sizes)]
        sc.pool.keep(sc.ids, first, [len(p) for p in paths], sum(paths, []))
        positions = [p + len(path) for p, path in zip(positions, paths)]
        # the last token's weights join the sums
        q1, o1, l1 = sc.buffers(2)
        sc.pool.extend(sc.ids, [1, 1], q1, o1, l1)
        old = [s.clone() for s in sums]
        sc.pool.weights(sc.ids, [1, 1], q1, l1, sums, old=sums, decay=1.0)
        torch.cuda.synchronize()
        for i in range(2):
            n = rows[i].shape[0]
            assert torch.equal(sc.held(sc.ids[i], n), rows[i]) and sc.pool.position(sc.ids[i]) == positions[i]
            w = given(name, rows[i], q1[i:i + 1], l1[i:i + 1])
            err = (sums[i][:, :n].double().cpu() - old[i][:, :n].double().cpu() - w).abs()
            assert (err <= 2.0 ** -11 * w + 2.0 ** -22 * (w + old[i][:, :n].double().cpu()) + 1e-30).all()
        full = [i for i in range(2) if rows[i].shape[0] > budget]
        if full:
            ws = [sums[i].cpu() for i in full]
            sc.pool.evict([sc.ids[i] for i in full], [200] * len(full), [sums[i] for i in full], new=[sums[i] for i in full],
                          first=4, last=16)
            for i, w in zip(full, ws):
                n = rows[i].shape[0]
                kept = [[heaviest(w[h, :n].tolist(), 200, 4, 16) for h in range(sc.hkv)]]
                rows[i] = kept_rows(name, rows[i][None], kept)[0].cuda()
                assert torch.equal(sc.held(sc.ids[i], 200), rows[i])
                assert (sums[i][:, 200:n] == 0).all()
    assert sc.pool.ctx_len(sc.ids[1]) < positions[1]
    rope.destroy()
    sc.close()


@pytest.mark.parametrize("name", ["gqa8x2d128", "mla16"])
def test_rows_that_lie_between_one_anothers(name):
    """One tensor for every request's numbers, requests inside layers: sums, choice and
    numbers as with tensors of their own."""
    print(f"[case] interleaved {name}", flush=True)
    layers, n, lens = 3, 3, [200, 77, 131]
    sc = Scene(name, lens, seed=8, layers=layers, room=10)
    forks = [sc.pool.open(sc.model, m + 10) for m in lens]
    sc.pool.fork(sc.ids, forks)
    q, _, lse = sc.buffers(30 * n)
    lse.fill_(3.0)
    t = max(lens)
    one, apart = torch.full((layers, n, sc.hkv, t), 7.0, device="cuda"), []
    slices = [one[:, i, :, :m] for i, m in enumerate(lens)]
    apart = [torch.full((layers, sc.hkv, m), 7.0, device="cuda") for m in lens]
    for layer in range(layers):
        sc.pool.weights(sc.ids, [30] * n, q, lse, slices, layer=layer)
        sc.pool.weights(sc.ids, [30] * n, q, lse, apart, layer=layer)
        sc.pool.weights(sc.ids, [30] * n, q, lse, slices, old=slices, decay=0.5, layer=layer)
        sc.pool.weights(sc.ids, [30] * n, q, lse, apart, old=apart, decay=0.5, layer=layer)
    for x, y in zip(slices, apart):
        assert torch.equal(x, y) and (y != 7).all()
    keep = [60, 77, 20]
    numbers = torch.full((layers, n, sc.hkv, t), -1, dtype=torch.int32, device="cuda")
    lists = [numbers[:, i, :, :k] for i, k in enumerate(keep)]
    own = [torch.full((layers, sc.hkv, k), -1, dtype=torch.int32, device="cuda") for k in keep]
    sc.pool.evict(sc.ids, keep, slices, new=slices, kept=lists, first=4, last=9)
    sc.pool.evict(forks, keep, apart, new=apart, kept=own, first=4, last=9)
    for i, (a, b, k) in enumerate(zip(sc.ids, forks, keep)):
        assert torch.equal(slices[i], apart[i]) and torch.equal(lists[i], own[i])
        assert torch.equal(sc.held(a, k, layers), sc.held(b, k, layers))
        assert (one[:, i, :, lens[i]:] == 7).all() and (numbers[:, i, :, k:] == -1).all()
    sc.ids += forks
    sc.close()


def test_two_graphs_of_sums_share_a_workspace():
    """Parts of rows in the pool's workspace: replays in turn, with an eager call between."""
    print("[case] two graphs", flush=True)
    sc = Scene("gqa8x2d128", [3000, 700], seed=9)
    sets = []
    stream = torch.cuda.Stream()
    for k, splits in ((300, 5), (64, 3)):
        q, _, lse = sc.buffers(2 * k)
        lse.fill_(2.0 + splits)
        new = [torch.zeros(sc.hkv, m, device="cuda") for m in (3000, 700)]
        call = lambda new=new, q=q, lse=lse, k=k, splits=splits: sc.pool.weights(sc.ids, [k, k], q, lse, new, num_splits=splits)
        with torch.cuda.stream(stream):
            call()
        stream.synchronize()
        want = [x.clone() for x in new]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call()
        sets.append((g, call, new, want))
    for turn in range(4):
        for g, call, new, want in sets:
            for x in new:
                x.fill_(-1.0)
            if turn == 2:
                call()
                for x, y in zip(new, want):
                    assert torch.equal(x, y)
                    x.fill_(-1.0)
            g.replay()
            torch.cuda.synchronize()
            for x, y in zip(new, want):
                assert torch.equal(x, y), turn
    sc.close()


def test_a_stream_of_their_own():
    """Sums, an eviction and kept tokens one behind the other on a side stream."""
    print("[case] side stream", flush=True)
    sc = Scene("gqa8x2d128", [2500], seed=10, room=50)
    b = sc.pool.open(sc.model, 2600)
    sc.pool.fork(sc.ids, [b])
    torch.cuda.synchronize()
    side, out = torch.cuda.Stream(), []
    q, _, lse = sc.buffers(40)
    lse.fill_(4.0)
    for rid, stream in ((sc.ids[0], torch.cuda.current_stream()), (b, side)):
        new = torch.zeros(1, sc.hkv, 2500, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            if stream is side:
                torch.cuda._sleep(2_000_000)
            sc.pool.weights([rid], [40], q, lse, [new])
            sc.pool.evict([rid], [900], [new], new=[new], first=5, last=40)
            sc.pool.keep([rid], [800], [30], list(range(0, 90, 3)))
            rows = sc.held(rid, 830)
        torch.cuda.synchronize()
        out.append((new, rows))
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
    sc.ids.append(b)
    sc.close()
