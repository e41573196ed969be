"""Forking and truncating requests on the CPU: page sharing, budgets,
reservations and refusals, against a model that counts pages by hand (no GPU: a
host-only pool does the bookkeeping)."""
import random

import numpy as np
import pytest

from paper_2606_24506_amd import crosspool as cpl

P = 4
ROW = dict(kind=cpl.CP_KIND_GQA, n_q_heads=1, n_kv_heads=1, head_dim=64)  # 256 bytes a token, 1 KiB a page


def pool(chunks=64, pages_per_chunk=8, **kw):
    return cpl.Pool(page_tokens=P, pool_bytes=chunks * pages_per_chunk * 1024, chunk_bytes=pages_per_chunk * 1024,
                    device=-1, **kw)


def grow(p, rid, n):
    p.append([rid], [n], None)


def test_fork_shares_whole_pages_and_copies_the_last():
    p = pool()
    m = p.register(**ROW)
    a, b, c = (p.open(m, 100) for _ in range(3))
    grow(p, a, 10)  # pages 0, 1 full, 2 with two tokens
    p.fork([a, a], [b, c], [10, 8])
    assert (p.ctx_len(b), p.ctx_len(c)) == (10, 8)
    pa, pb, pc = p.pages(a), p.pages(b), p.pages(c)
    assert list(pb[:2]) == list(pa[:2]) and pb[2] != pa[2]
    assert list(pc) == list(pa[:2])
    s = p.stats()
    assert s["pages_used"] == 4  # 3 of a, b's last
    # what all three may still take, and what is there
    assert s["pages_reserved"] == 4 + (25 - 3) + (25 - 3) + (25 - 2)
    # each goes on in pages of its own
    grow(p, c, 1)
    grow(p, a, 3)
    grow(p, b, 1)
    pa, pb, pc = p.pages(a), p.pages(b), p.pages(c)
    assert len(set(pa[2:]) | set(pb[2:]) | set(pc[2:])) == len(pa[2:]) + len(pb[2:]) + len(pc[2:])
    p.close(a)
    assert list(p.pages(b)[:2]) == list(pa[:2])  # still shown by b and c
    p.close(b)
    p.close(c)
    assert p.stats()["pages_used"] == p.stats()["pages_reserved"] == p.stats()["chunks_used"] == 0
    p.destroy()


def test_truncate_gives_pages_back_and_owns_the_last():
    p = pool()
    m = p.register(**ROW)
    a, b = p.open(m, 100), p.open(m, 100)
    grow(p, a, 21)
    p.fork([a], [b])
    before = p.pages(a)
    p.truncate([b], [6])  # inside page 1, which a shows too
    pb = p.pages(b)
    assert pb[0] == before[0] and pb[1] != before[1] and len(pb) == 2
    assert list(p.pages(a)) == list(before)
    p.truncate([a], [8])
    assert list(p.pages(a)) == list(before[:2])
    assert p.stats()["pages_used"] == 3
    p.truncate([a, b], [0, 0])
    s = p.stats()
    assert (p.ctx_len(a), p.ctx_len(b)) == (0, 0)
    assert s["pages_used"] == 0 and s["pages_reserved"] == 50 and s["chunks_used"] == 0
    grow(p, a, 100)
    grow(p, b, 100)
    with pytest.raises(cpl.CrossPoolError):
        grow(p, a, 1)
    for r in (a, b):
        p.close(r)
    p.destroy()


def test_sharing_gives_budget_back_and_truncation_takes_it():
    p = pool(chunks=2, pages_per_chunk=8)  # 16 pages
    m = p.register(**ROW)
    a = p.open(m, 8 * P)
    b = p.open(m, 8 * P)
    grow(p, a, 8 * P)
    with pytest.raises(cpl.CrossPoolError) as e:
        p.open(m, P)
    assert e.value.status == cpl.CP_ENOSPC
    p.fork([a], [b])
    c = p.open(m, 8 * P)  # b's eight pages are a's
    assert p.stats()["pages_reserved"] == 16
    with pytest.raises(cpl.CrossPoolError) as e:
        p.truncate([b], [2])  # b's reservation would need pages of its own again
    assert e.value.status == cpl.CP_ENOSPC
    assert p.ctx_len(b) == 8 * P and list(p.pages(b)) == list(p.pages(a))
    p.close(a)  # b alone shows them: they count for b
    assert p.stats()["pages_reserved"] == 16
    p.truncate([b], [2])
    grow(p, b, 8 * P - 2)
    grow(p, c, 8 * P)
    assert p.stats()["pages_used"] == 16
    for r in (b, c):
        p.close(r)
    p.destroy()


def test_two_models_keep_their_budgets():
    p = pool(chunks=4, pages_per_chunk=8)
    m1, m2 = p.register(**ROW), p.register(**dict(ROW, n_q_heads=2, n_kv_heads=2))  # 4 pages a chunk
    a, b = p.open(m1, 16 * P), p.open(m1, 8 * P)
    c = p.open(m2, 4 * P)
    grow(p, a, 8 * P + 1)
    with pytest.raises(cpl.CrossPoolError):
        p.open(m2, 4 * P)  # 24 and 4 pages: all four chunks
    p.fork([a], [b], [8 * P])  # 16 and 4
    d = p.open(m2, 4 * P)
    grow(p, c, 4 * P)
    with pytest.raises(cpl.CrossPoolError) as e:
        p.fork([a], [c])
    assert e.value.status == cpl.CP_EINVAL
    for r in (a, b, c, d):
        p.close(r)
    assert p.stats()["chunks_used"] == 0
    p.destroy()


def test_one_call_truncates_all_users_of_a_page():
    """Users that cut inside, drop and keep the same shared page in one call."""
    p = pool()
    m = p.register(**ROW)
    ids = [p.open(m, 40) for _ in range(4)]
    grow(p, ids[0], 16)
    p.fork([ids[0]] * 3, ids[1:])
    p.truncate(ids, [6, 0, 7, 12])
    pg = [list(p.pages(r)) for r in ids]
    assert len(pg[0]) == 2 and len(pg[2]) == 2 and len(pg[3]) == 3
    assert pg[0][0] == pg[2][0] == pg[3][0]
    assert len({pg[0][1], pg[2][1], pg[3][1]}) == 3
    assert p.stats()["pages_used"] == 1 + 3 + 1
    for r in ids:
        p.close(r)
    assert p.stats()["chunks_used"] == 0
    p.destroy()


@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("placement", [0, 7])
@pytest.mark.parametrize("backing", [cpl.CP_BACKING_BUFFER, cpl.CP_BACKING_VIRTUAL])
def test_random_calls_against_a_page_count(layers, placement, backing):
    """Random opens, appends, forks, truncations and closes: what a request
    shows is what a copy would, no two write the same page, and the counters
    are those of the distinct pages."""
    rng = random.Random(layers * 10 + placement + backing)
    p = pool(chunks=40, placement_seed=placement, backing=backing)
    m = p.register(**ROW, n_layers=layers)
    live = {}  # id -> (reserved tokens, list of (layer pages)) by content
    content = {}  # page entry -> list of token stamps
    held = {}  # id -> token stamps
    stamp = 0

    def check():
        pages = set()
        room = 0
        for r, (cap, _) in live.items():
            assert p.ctx_len(r) == len(held[r])
            n = -(-len(held[r]) // P)
            tab = p.pages(r, 0, n, layers) if n else np.zeros((layers, 0), np.uint32)
            tab = np.asarray(tab).reshape(layers, n)
            for l in range(layers):
                for k in range(n):
                    mine = [(l, s) for s in held[r][k * P:(k + 1) * P]]
                    assert content[tab[l, k]][:len(mine)] == mine, (r, l, k)
                    pages.add(int(tab[l, k]))
            room += (-(-cap // P) - n) * layers
        s = p.stats()
        assert s["pages_used"] == len(pages)
        assert s["pages_reserved"] == len(pages) + room

    def write(r, start):
        """The new tokens' stamps go into the pages they lie in, as the copy
        kernels do with rows."""
        n = -(-len(held[r]) // P)
        tab = np.asarray(p.pages(r, 0, n, layers)).reshape(layers, n)
        for i in range(start, len(held[r])):
            for l in range(layers):
                page = content.setdefault(int(tab[l, i // P]), [None] * P)
                page[i % P] = (l, held[r][i])

    def copied(src_tab, r, n_tok):
        """Forked or cut inside a page: its tokens are copied to the own page."""
        n = -(-n_tok // P)
        if n_tok % P:
            tab = np.asarray(p.pages(r, 0, n, layers)).reshape(layers, n)
            for l in range(layers):
                a, b = int(src_tab[l][n - 1]), int(tab[l, n - 1])
                if a != b:
                    content[b] = list(content[a][:n_tok % P]) + [None] * (P - n_tok % P)

    def table(r):
        n = -(-len(held[r]) // P)
        return np.asarray(p.pages(r, 0, n, layers)).reshape(layers, n).tolist() if n else [[] for _ in range(layers)]

    for step in range(700):
        do = rng.choice(["open", "append", "append", "fork", "fork", "truncate", "truncate", "close"])
        ids = list(live)
        try:
            if do == "open":
                cap = rng.randint(1, 60)
                r = p.open(m, cap)
                live[r], held[r] = (cap, None), []
            elif do == "append" and ids:
                r = rng.choice(ids)
                n = rng.randint(0, 12)
                before = len(held[r])
                p.append([r], [n], None)
                held[r] += [stamp + i for i in range(n)]
                stamp += n
                if n:
                    write(r, before)
            elif do == "fork" and ids:
                src = rng.choice(ids)
                dst = [r for r in ids if r != src and not held[r]][:2]
                if dst:
                    toks = [rng.randint(0, len(held[src])) for _ in dst]
                    tab = table(src)
                    p.fork([src] * len(dst), dst, toks)
                    for r, n in zip(dst, toks):
                        held[r] = held[src][:n]
                        copied(tab, r, n)
            elif do == "truncate" and ids:
                some = rng.sample(ids, min(len(ids), rng.randint(1, 3)))
                to = [rng.randint(0, len(held[r])) for r in some]
                tabs = [table(r) for r in some]
                p.truncate(some, to)
                for r, n, tab in zip(some, to, tabs):
                    held[r] = held[r][:n]
                for r, n, tab in zip(some, to, tabs):
                    copied(tab, r, n)
            elif do == "close" and len(ids) > 3:
                r = rng.choice(ids)
                p.close(r)
                del live[r], held[r]
        except cpl.CrossPoolError as e:
            assert e.status in (cpl.CP_ENOSPC, cpl.CP_EINVAL), e
        check()
    for r in list(live):
        p.close(r)
    s = p.stats()
    assert s["pages_used"] == s["pages_reserved"] == s["chunks_used"] == 0
    p.destroy()


def test_admitted_requests_can_always_fill_their_reservations():
    """After forks and truncations, as at admission."""
    for seed in range(30):
        rng = random.Random(seed)
        p = pool(chunks=6, placement_seed=seed)
        m = p.register(**ROW)
        caps = {}
        for _ in range(60):
            try:
                do = rng.random()
                if do < 0.3:
                    c = rng.randint(1, 80)
                    caps[p.open(m, c)] = c
                elif caps and do < 0.5:
                    r = rng.choice(list(caps))
                    p.append([r], [rng.randint(0, 10)], None)
                elif len(caps) > 1 and do < 0.75:
                    a, b = rng.sample(list(caps), 2)
                    p.fork([a], [b], None)
                elif caps and do < 0.95:
                    r = rng.choice(list(caps))
                    p.truncate([r], [rng.randint(0, p.ctx_len(r))])
                elif caps:
                    r = rng.choice(list(caps))
                    p.close(r)
                    del caps[r]
            except cpl.CrossPoolError as e:
                assert e.status in (cpl.CP_ENOSPC, cpl.CP_EINVAL), e
        for r, c in caps.items():
            p.append([r], [-(-c // P) * P - p.ctx_len(r)], None)
        for r in caps:
            p.close(r)
        assert p.stats()["chunks_used"] == 0
        p.destroy()


def refused(fn, *args, status=cpl.CP_EINVAL):
    with pytest.raises(cpl.CrossPoolError) as e:
        fn(*args)
    assert e.value.status == status, e.value


def test_refusals_change_nothing():
    p = pool()
    m, m2 = p.register(**ROW), p.register(**ROW)
    a, b, c, d = p.open(m, 40), p.open(m, 8), p.open(m, 40), p.open(m2, 40)
    grow(p, a, 20)
    grow(p, c, 3)
    before = p.stats()
    refused(p.fork, [a], [99])
    refused(p.fork, [99], [b])
    refused(p.fork, [a], [a])
    refused(p.fork, [a, b], [b, c])    # b twice
    refused(p.fork, [a, a], [b, b])
    refused(p.fork, [a], [c])          # not empty
    refused(p.fork, [a], [d])          # another model
    refused(p.fork, [a], [b])          # 20 tokens do not fit 8
    refused(p.fork, [a], [b], [21])
    refused(p.fork, [a], [b], [-1])
    refused(p.truncate, [a], [21])
    refused(p.truncate, [a], [-1])
    refused(p.truncate, [a, a], [1, 2])
    refused(p.truncate, [a, c], [1, 4])  # the second refused: neither is cut
    refused(p.truncate, [77], [0])
    assert p.stats() == before and p.ctx_len(a) == 20
    p.fork([a], [b], [8])
    p.fork([], [])
    p.truncate([], [])
    p.truncate([a], [20])
    for r in (a, b, c, d):
        p.close(r)
    p.destroy()


def test_rope_and_extend_refusals():
    """What the new calls refuse, without a GPU."""
    for kw in (dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=1026), dict(rot_dim=8, base=0.0),
               dict(rot_dim=8, scaling=cpl.CP_ROPE_LINEAR, factor=0.0), dict(rot_dim=2, scaling=cpl.CP_ROPE_NTK, factor=2.0),
               dict(rot_dim=8, scaling=cpl.CP_ROPE_PARTS, factor=2.0), dict(rot_dim=8, scaling=9), dict(rot_dim=8, layout=2),
               dict(rot_dim=8, scaling=cpl.CP_ROPE_TABLE), dict(rot_dim=4, scaling=cpl.CP_ROPE_TABLE, table=[1.0, float("inf")]),
               dict(rot_dim=8, magnitude=float("nan")), dict(rot_dim=8, device=1000)):
        with pytest.raises(cpl.CrossPoolError) as e:
            cpl.cp_rope_create(**{"device": -1, **kw})
        assert e.value.status == cpl.CP_EINVAL
    rope = cpl.Rope(8, device=-1)
    one = cpl.cp_rope_tensor(4096, 4096, 8, 8, 8, 8, 1, 8, 0, cpl.CP_ROPE_BF16)

    def apply(t, n=1, tokens=2, first=0):
        arr = (cpl.cp_rope_tensor * max(1, n))(*[t] * n)
        rc = cpl.LIB.cp_rope_apply(rope.handle, n, arr, tokens, None, first, 0, None)
        if rc:
            raise cpl.CrossPoolError(rc, cpl.LIB.cp_last_error().decode())

    def changed(**kw):
        t = cpl.cp_rope_tensor.from_buffer_copy(one)
        for k, v in kw.items():
            setattr(t, k, v)
        return t

    refused(apply, one, status=cpl.CP_ESTATE)  # all of it right, but no device
    for kw in (dict(src=None), dict(dst=None), dict(offset=1), dict(offset=-1), dict(width=7), dict(heads=0),
               dict(dtype=2), dict(src_token=-8), dict(dst_token=4), dict(src=4097), dict(heads=2, dst_head=4),
               dict(src_token=16)):  # the last: in place with other strides
        refused(apply, changed(**kw))
    refused(apply, one, 0)
    refused(apply, one, 17)
    refused(apply, one, 1, -1)
    refused(apply, one, 1, 1, 1 << 60)
    p = pool()
    m = p.register(**ROW)
    a = p.open(m, 40)
    grow(p, a, 4)
    wide = cpl.Rope(66, device=-1)
    refused(p.append_rope, [a], [1], None, wide)
    refused(p.append_rope, [a], [100], None, rope)
    p.append_rope([a], [2], None, rope)  # a host-only pool keeps its books
    assert p.ctx_len(a) == 6
    refused(p.extend, [a], [1], None, None, None, status=cpl.CP_ESTATE)
    refused(p.extend_step, [a], [1], None, None, None, None, status=cpl.CP_ESTATE)
    p.close(a)
    p.destroy()


def test_rows_of_a_rotation_that_overlap_are_refused():
    rope = cpl.Rope(8, device=-1)

    def refused(tokens, heads, token, head, width=16):
        t = (cpl.cp_rope_tensor * 1)()
        t[0] = cpl.cp_rope_tensor(4096, 1 << 30, width, width * tokens, token, head, heads, width, 0, cpl.CP_ROPE_BF16)
        t.tokens = tokens
        with pytest.raises(cpl.CrossPoolError) as e:
            cpl.cp_rope_apply(rope.handle, t)
        return e.value.status != cpl.CP_ESTATE  # (a host-only rotation refuses sound calls too, last)

    for tokens, heads, width in ((1, 1, 16), (1, 5, 16), (5, 1, 16), (4, 3, 16), (2, 7, 9), (6, 6, 16)):
        for token in (0, 1, 9, 15, 16, 17, 24, 32, 40, 48, 80, 112):
            for head in (0, 8, 15, 16, 20, 32, 33, 48, 64, 80, 1 << 61):
                at = sorted(t * token + h * head for t in range(tokens) for h in range(heads))
                meet = any(b - a < width for a, b in zip(at, at[1:]))
                assert refused(tokens, heads, token, head, width) == meet, (tokens, heads, token, head, width)
    rope.destroy()


def test_tensors_of_attention_off_the_gpu_are_refused():
    import torch

    host, where = torch.zeros(2, 4), 4096
    dev = torch.zeros(3, dtype=torch.int32)
    for kw in (dict(q=host), dict(out=host), dict(lse=host), dict(slopes=host), dict(doc_begin=dev)):
        with pytest.raises(ValueError):
            cpl.cp_attn_extend(None, [0], [3], **{**dict(q=where, out=where, lse=where), **kw})
        with pytest.raises(ValueError):
            cpl.cp_attn_extend_step(None, [0], [3], **{**dict(rows=where, q=where, out=where, lse=where), **kw})
    with pytest.raises(ValueError):
        cpl.cp_attn_extend_step(None, [0], [3], host, where, where, where)
    t = (cpl.cp_rope_tensor * 1)()
    t.tokens = 3
    with pytest.raises(ValueError):
        cpl.cp_rope_apply(None, t, positions=dev)
