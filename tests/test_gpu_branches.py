"""A prompt and its branches on the GPU: forked and truncated requests hold the
rows they should, chunks are placed and attended layer by layer, and the
operators run together as a serving program calls them."""
import numpy as np
import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, Scene, attend, bits, check, rounds_to_16_bits, shape, turn, turn_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["gqa8x2d128", "mla16", "gqa6x2d64", "mla4l128r40"])
@pytest.mark.parametrize("page_tokens", [16, 64, 96])
@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("kw", [{}, dict(backing=cpl.CP_BACKING_VIRTUAL), dict(device_pages=1)])
def test_forks_and_truncations_hold_the_rows(name, page_tokens, layers, kw):
    print(f"[case] fork {name} P{page_tokens} layers {layers} {kw}", flush=True)
    sc = Scene(name, [0], page_tokens=page_tokens, seed=30, room=400, layers=layers, pool_bytes=256 << 20, **kw)
    p, src = sc.pool, sc.ids[0]
    rows = sc.normal(layers, 333, sc.row)
    p.append([src], [333], rows)
    want = {src: rows}
    lens = [0, 1, page_tokens, page_tokens * 2 + 3, 333]
    dst = [p.open(sc.model, 400) for _ in lens]
    sc.ids += dst
    p.fork([src] * len(dst), dst, lens)
    for r, n in zip(dst, lens):
        want[r] = rows[:, :n]

    def same():
        for r, w in want.items():
            assert p.ctx_len(r) == w.shape[1]
            got = sc.held(r, w.shape[1], layers)
            assert (bits(got).reshape(-1) == bits(w).reshape(-1)).all(), r

    same()

    def append(r, n):
        new = sc.normal(layers, n, sc.row)
        p.append([r], [n], new)
        want[r] = torch.cat([want[r], new], 1)

    for r in [src] + dst:  # all go on, in pages of their own
        append(r, 5)
    same()
    # the parent and two children cut inside shared pages, one call
    cut = [src, dst[3], dst[4]]
    to = [page_tokens + 2, page_tokens // 2, page_tokens + 2]
    p.truncate(cut, to)
    for r, n in zip(cut, to):
        want[r] = want[r][:, :n]
    same()
    for r in cut:
        append(r, page_tokens + 1)
    same()
    p.fork([dst[4], dst[4]], [d for d in [p.open(sc.model, 400), p.open(sc.model, 400)] if not sc.ids.append(d)])
    for r in sc.ids[-2:]:
        want[r] = want[dst[4]]
    torch.cuda.synchronize()
    p.close(src)  # its children keep what they show
    sc.ids.remove(src)
    del want[src]
    same()
    append(sc.ids[-1], 70)
    same()
    sc.close()


def test_fork_of_many_planes_takes_several_launches():
    sc = Scene("mla4l64r0", [0], page_tokens=16, seed=31, room=100, layers=50, pool_bytes=256 << 20)
    rows = sc.normal(50, 37, sc.row)
    sc.pool.append(sc.ids, [37], rows)
    dst = [sc.pool.open(sc.model, 100) for _ in range(3)]
    sc.pool.fork(sc.ids * 3, dst)
    for d in dst:
        assert (bits(sc.held(d, 37, 50)) == bits(rows)).all()
    sc.ids += dst
    sc.close()


@pytest.mark.parametrize("kw", [{}, dict(device_pages=1)])
@pytest.mark.parametrize("name", ["gqa8x2d128", "mla16"])
def test_chunks_go_layer_by_layer(name, kw):
    """A prompt in chunks through three layers, keys rotated as they are
    placed; single tokens by the decode step in between; cursors and refusals."""
    L = 3
    sc = Scene(name, [0, 0], page_tokens=32, seed=32, room=600, layers=L, **kw)
    p = sc.pool
    rot = 64
    rope = cpl.Rope(rot, layout="interleaved")
    want = [[torch.zeros(0, sc.row, dtype=torch.bfloat16) for _ in range(L)] for _ in sc.ids]
    for step, n_new in enumerate([[100, 3], [45, 0], [1, 130], [0, 0]]):
        total = sum(n_new)
        for l in range(L):
            assert [p.cursor(r) for r in sc.ids] == [(l, n if l else 0) for n in n_new]
            rows = sc.normal(max(1, total), sc.row)
            q, out, lse = sc.buffers(max(1, total))
            p.extend_step(sc.ids, n_new, rows, q, out, lse, rope=rope, window=64 if l == 1 else 0)
            torch.cuda.synchronize()
            at = 0
            for i, n in enumerate(n_new):
                base = want[i][l].shape[0]
                new = turn_rows(name, rows[at:at + n], rope.angles(), torch.arange(base, base + n), "interleaved")
                want[i][l] = torch.cat([want[i][l], new.bfloat16()])
                if n:
                    # what was stored may round the other way: attend over the stored rows
                    ref = attend(name, stored(sc, i, l, base + n), q[at:at + n], window=64 if l == 1 else 0)
                    check(out[at:at + n], lse[at:at + n], ref, rounds_to_16_bits(name, n), f"step {step} layer {l}")
                at += n
            if l + 1 < L and max(n_new) > 1:
                for call in (lambda: p.append(sc.ids, [1, 1], rows), lambda: p.truncate(sc.ids, [0, 0]),
                             lambda: p.extend_step(sc.ids, [n + 1 for n in n_new], rows, q, out, lse)):
                    with pytest.raises(cpl.CrossPoolError) as e:
                        call()
                    assert e.value.status == cpl.CP_EINVAL
        assert [p.ctx_len(r) for r in sc.ids] == [w[0].shape[0] for w in want]
        # a token by the decode step, through the same layers
        for l in range(L):
            rows = sc.normal(2, sc.row)
            q, out, lse = sc.buffers(2)
            p.decode_step(sc.ids, [1, 1], rows, q, out, lse)
            for i in range(2):
                want[i][l] = torch.cat([want[i][l], rows[i:i + 1].cpu()])
    for i, r in enumerate(sc.ids):
        n = want[i][0].shape[0]
        got = sc.held(r, n, L).double().cpu()
        exp = torch.stack(want[i]).double()
        assert ((got - exp).abs() <= 2.0 ** -7 * exp.abs() + 1e-6).all()  # a step apart where a rounding is close
    rope.destroy()
    sc.close()


def stored(sc, i, layer, n):
    """Rows of a plane while the chunk is in flight (not committed: read through
    the page table)."""
    torch.cuda.synchronize()
    r = sc.ids[i]
    tab = sc.pool.pages(r, 0, -(-n // sc.pool.page_tokens), 3)[layer]
    P, out = sc.pool.page_tokens, []
    base = page_memory(sc)
    for k, pte in enumerate(tab):
        page = base[int(pte) * 128:int(pte) * 128 + P * sc.row]
        if GEOMS[sc.name]["kind"] == cpl.CP_KIND_MLA:
            out.append(page.view(P, sc.row))
        else:
            out.append(page.view(sc.hkv, 2, P, sc.dk).permute(2, 1, 0, 3).reshape(P, sc.row))
    return torch.cat(out)[:n]


def page_memory(sc):
    return sc.mem


@pytest.fixture(autouse=True)
def own_memory(monkeypatch):
    """Scenes of these tests sit in memory that the test can read, unless the
    pool maps its own."""
    init = Scene.__init__

    def with_memory(self, *a, **k):
        if k.get("backing") != cpl.CP_BACKING_VIRTUAL:
            k.setdefault("fill", float("nan"))
        init(self, *a, **k)

    monkeypatch.setattr(Scene, "__init__", with_memory)


@pytest.mark.parametrize("name", ["gqa8x2d128", "mla16", "gqa6x2d64"])
def test_a_prompt_and_its_branches(name):
    """As a serving program runs them: the prompt is placed in two chunks
    (queries rotated by cp_rope_apply, keys on the way in), forked into branches that
    take tokens of their own, drafted tokens are dropped, a branch takes another
    parent, and the decode call reads the result."""
    sc = Scene(name, [0], page_tokens=64, seed=33, room=600, pool_bytes=128 << 20)
    p, dk = sc.pool, sc.dk
    mla = GEOMS[name]["kind"] == cpl.CP_KIND_MLA
    rot, off = 64, sc.dv if mla else 0
    rope = cpl.Rope(rot, layout="half", scaling="parts", factor=4.0, orig_len=128)
    slopes = torch.linspace(0.02, 0.3, sc.hq, device="cuda")
    opts = dict(softcap=20.0, window=300, slopes=slopes)

    def step(ids, n_new):
        total = sum(n_new)
        rows = sc.normal(total, sc.row, sigma=0.7)
        q, out, lse = sc.buffers(total)
        pos = torch.cat([torch.arange(p.ctx_len(r), p.ctx_len(r) + n) for r, n in zip(ids, n_new)]).to("cuda", torch.int32)
        before = [sc.held(r, p.ctx_len(r)) for r in ids]
        turned = torch.empty_like(q)
        rope.apply(cpl.rope_parts([(q, turned)], offset=off), pos)
        p.extend_step(ids, n_new, rows, turned, out, lse, rope=rope, **opts)
        torch.cuda.synchronize()
        want_q = q.double().cpu()
        want_q[..., off:off + rot] = turn(q[..., off:off + rot], rope.angles(), pos, "half")
        assert ((turned.double().cpu() - want_q).abs() <= 2.0 ** -8 * want_q.abs() + 1e-5).all()
        at = 0
        for r, n, old in zip(ids, n_new, before):
            got = sc.held(r, p.ctx_len(r))
            assert (bits(got[:len(old)]) == bits(old)).all()
            new = turn_rows(name, rows[at:at + n], rope.angles(), pos[at:at + n], "half")
            assert ((got[len(old):].double().cpu() - new).abs() <= 2.0 ** -8 * new.abs() + 1e-5).all()
            check(out[at:at + n], lse[at:at + n], attend(name, got, turned[at:at + n], **opts),
                  rounds_to_16_bits(name, n), f"{name} request {r}")
            at += n

    root = sc.ids[0]
    step([root], [150])
    step([root], [61])
    kids = [p.open(sc.model, 600) for _ in range(3)]
    sc.ids += kids
    p.fork([root] * 3, kids, [211, 211, 128])
    step(kids, [1, 6, 2])
    step(kids + [root], [1, 1, 1, 4])
    p.truncate(kids[:2], [212, 214])  # drafted tokens that were not accepted
    step(kids, [3, 3, 3])
    p.truncate([kids[2]], [0])  # a beam takes another parent
    p.fork([kids[1]], [kids[2]])
    step(kids, [1, 1, 1])
    q, out, lse = sc.buffers(4)
    p.decode(sc.ids, q, out, lse)
    torch.cuda.synchronize()
    for i, r in enumerate(sc.ids):
        ref = attend(name, sc.held(r, p.ctx_len(r)), q[i:i + 1])
        assert ((out[i].double().cpu() - ref[0][0]).abs() <= 2.0 ** -8 * ref[0][0].abs() + 2.0 ** -7 * ref[2][0]).all()
        assert (lse[i].double().cpu() - ref[1][0]).abs().max() <= 1e-3
    rope.destroy()
    sc.close()


def test_a_refused_step_changes_nothing():
    sc = Scene("gqa8x2d128", [100, 30], seed=34, room=10)
    other = sc.pool.register(**GEOMS["gqa6x2d64"])
    alien = sc.pool.open(other, 10)
    q, out, lse = sc.buffers(8)
    rows = sc.normal(8, sc.row)
    before = sc.pool.stats()
    rope = cpl.Rope(130)

    def bad(**kw):
        args = dict(ids=sc.ids, n=[1, 2], rows=rows, q=q, out=out, lse=lse)
        opts = {k: v for k, v in kw.items() if k not in args}
        args.update({k: v for k, v in kw.items() if k in args})
        with pytest.raises(cpl.CrossPoolError) as e:
            sc.pool.extend_step(args["ids"], args["n"], args["rows"], args["q"], args["out"], args["lse"], **opts)
        assert e.value.status == cpl.CP_EINVAL, e.value

    bad(n=[-1, 2])
    bad(n=[200, 1])  # past the reservation
    bad(rows=None)
    bad(q=None)
    bad(lse=None)
    bad(ids=[sc.ids[0], sc.ids[0]])
    bad(ids=[sc.ids[0], alien])
    bad(ids=[], n=[])
    bad(softcap=-1.0)
    bad(softcap=float("nan"))
    bad(window=-1)
    bad(num_splits=-1)
    bad(path=cpl.CP_PATH_MFMA)
    bad(prefix=[0, -1])
    bad(rope=rope)
    bad(q=q.data_ptr() + 2)
    bad(out=out.data_ptr() + 4)
    with pytest.raises(cpl.CrossPoolError):
        sc.pool.extend(sc.ids, [101, 1], q, out, lse)
    assert sc.pool.stats() == before and sc.pool.ctx_len(sc.ids[0]) == 100
    torch.cuda.synchronize()
    assert (out == 7).all()
    sc.pool.close(alien)
    sc.close()


def test_a_capped_workspace_bounds_the_ranges():
    """Ranges are given up to stay under the pool's cap, and forced ones refused."""
    sc = Scene("gqa8x2d128", [5000], seed=35, max_workspace_bytes=40000)
    q, out, lse = sc.buffers(1)
    sc.pool.extend(sc.ids, [1], q, out, lse)
    torch.cuda.synchronize()
    check(out, lse, attend(sc.name, sc.rows[0], q), False, "capped")
    with pytest.raises(cpl.CrossPoolError) as e:
        sc.pool.extend(sc.ids, [1], q, out, lse, num_splits=30)
    assert e.value.status == cpl.CP_ENOMEM
    sc.close()
