"""A truncation takes no chunk of the budget that it does not fill (CPU)."""
import random

import pytest

from paper_2606_24506_amd import crosspool as cpl

P = 4
ROW = dict(kind=cpl.CP_KIND_GQA, n_q_heads=1, n_kv_heads=1, head_dim=64)  # 1 KiB a page


def pool(chunks, **kw):
    return cpl.Pool(page_tokens=P, pool_bytes=chunks * 8 * 1024, chunk_bytes=8 * 1024, device=-1, **kw)


@pytest.mark.parametrize("seed", [0, 3])
def test_users_of_one_page_take_no_chunk_for_each(seed):
    """Two requests cut inside a page that only they show: one copy, which the chunk has
    room for, though a copy for each would not fit."""
    p = pool(2, placement_seed=seed)
    m, other = p.register(**ROW), p.register(**ROW)
    a, b = p.open(m, 28), p.open(m, 28)
    p.append([a], [28], None)
    p.fork([a], [b])
    p.truncate([a, b], [26, 26])
    s = p.stats()
    assert (s["pages_used"], s["pages_reserved"], s["chunks_used"]) == (8, 8, 1)
    c = p.open(other, 32)  # the other chunk
    p.append([c], [32], None)
    for r in (a, b, c):
        p.close(r)
    assert p.stats()["chunks_used"] == 0
    p.destroy()


@pytest.mark.parametrize("seed", range(20))
def test_no_chunk_is_held_empty(seed):
    """Random calls of two models: as many chunks as pages in use fill, one by one."""
    rng = random.Random(seed)
    p = pool(20, placement_seed=seed % 3)
    models = [p.register(**ROW), p.register(**dict(ROW, n_q_heads=2, n_kv_heads=2))]
    live = {}
    for _ in range(400):
        do = rng.choice(["open", "append", "fork", "fork", "truncate", "truncate", "truncate", "close"])
        ids = list(live)
        try:
            if do == "open":
                m = rng.choice(models)
                live[p.open(m, rng.randint(1, 40))] = m
            elif do == "append" and ids:
                p.append([rng.choice(ids)], [rng.randint(0, 9)], None)
            elif do == "fork" and ids:
                src = rng.choice(ids)
                dst = [r for r in ids if r != src and live[r] == live[src] and p.ctx_len(r) == 0][:3]
                p.fork([src] * len(dst), dst)
            elif do == "truncate" and ids:
                some = rng.sample(ids, min(len(ids), rng.randint(1, 4)))
                least = min(p.ctx_len(r) for r in some)
                p.truncate(some, [rng.randint(0, least)] * len(some))
            elif do == "close" and len(ids) > 3:
                r = rng.choice(ids)
                p.close(r)
                del live[r]
        except cpl.CrossPoolError as e:
            assert e.status in (cpl.CP_ENOSPC, cpl.CP_EINVAL), e
        used = set()
        for r in live:
            n = -(-p.ctx_len(r) // P)
            used |= {int(x) // 32 for x in p.pages(r).reshape(-1)[:n]}  # entries count 256 bytes: 32 a chunk
        assert p.stats()["chunks_used"] == len(used)
    for r in live:
        p.close(r)
    assert p.stats()["chunks_used"] == 0
    p.destroy()
