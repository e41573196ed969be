"""Requests cut to some of their tokens while the device is behind the host, and in pools
whose budget has no page to spare: rows bit for bit."""
import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, shape

pytestmark = pytest.mark.gpu

NAME, P = "gqa6x2d64", 4
HQ, HKV, DK, DV, ROW, _ = shape(NAME)


def normal(gen, *size):
    return torch.empty(*size, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def held(p, r, n, layers=1):
    out = torch.zeros(layers, n, ROW, dtype=torch.bfloat16, device="cuda")
    p.gather(r, 0, n, out)
    return out


def behind():
    """Some 30 ms of work on the stream."""
    a = torch.ones(8192, 8192, dtype=torch.bfloat16, device="cuda")
    for _ in range(30):
        a @ a


def test_a_fork_keeps_a_prompt_that_is_evicted_behind_other_work():
    """The entries of 2,000 new pages (1,000 in each layer) are on their way while the pages are shared, replaced
    and shared again."""
    print("[case] append, fork, evict, fork, evict behind other work", flush=True)
    layers, n = 2, 4000
    gen = torch.Generator(device="cuda").manual_seed(1)
    chunk = 16 * P * 2 * ROW
    p = cpl.Pool(page_tokens=P, pool_bytes=600 * chunk, chunk_bytes=chunk, device=0)
    m = p.register(**GEOMS[NAME], n_layers=layers)
    a, b, c = (p.open(m, n) for _ in range(3))
    rows = normal(gen, layers, n, ROW)
    w = torch.rand(layers, HKV, n, generator=torch.Generator().manual_seed(2)).cuda()
    new, kept = torch.zeros_like(w), torch.zeros(layers, HKV, 2400, dtype=torch.int32, device="cuda")
    last = torch.zeros(layers, HKV, 2000, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    behind()
    p.append([a], [n], rows)
    p.fork([a], [b])
    p.evict([a], [2400], [w], new=[new], kept=[kept])
    p.fork([a], [c])
    p.evict([a], [2000], [new[..., :2400]], kept=[last])
    order = w.argsort(-1, descending=True).cpu()
    assert torch.equal(held(p, b, n, layers), rows)

    def cut(of, places):  # rows of the tokens that stay, per layer and KV head
        x = of.view(layers, -1, 2, HKV, DK)
        at = places.long()
        return torch.stack([torch.stack([x[l][at[l, h]][:, :, h] for h in range(HKV)], 2) for l in range(layers)]).view(
            layers, -1, ROW)

    want = order[..., :2400].sort(-1).values.cuda()
    assert torch.equal(kept.long(), want)
    assert torch.equal(held(p, c, 2400, layers), cut(rows, want))
    assert torch.equal(held(p, a, 2000, layers), cut(cut(rows, want), last))
    assert torch.equal(want.gather(-1, last.long()), order[..., :2000].sort(-1).values.cuda())
    for r in (a, b, c):
        p.close(r)
    p.destroy()


def test_drafts_dropped_and_placed_again_behind_other_work():
    """Steps, cuts and steps of two requests in turn, whose new pages change places."""
    print("[case] steps and cuts behind other work", flush=True)
    layers, n, new = 3, 6, 9
    gen = torch.Generator(device="cuda").manual_seed(3)
    chunk = 8 * P * 2 * ROW
    p = cpl.Pool(page_tokens=P, pool_bytes=200 * chunk, chunk_bytes=chunk, device=0)
    m = p.register(**GEOMS[NAME], n_layers=layers)
    ids = [p.open(m, 200) for _ in range(2)]
    rows = [normal(gen, layers, n, ROW) for _ in ids]
    p.append(ids, [n] * 2, torch.cat([x.view(-1) for x in rows]))
    steps = [[normal(gen, new, ROW) for _ in ids] for _ in range(4 * layers)]
    q = normal(gen, 2 * new, HQ, DK)
    o, lse = torch.zeros(2 * new, HQ, DV, dtype=torch.bfloat16, device="cuda"), torch.zeros(2 * new, HQ, device="cuda")
    got = []
    torch.cuda.synchronize()
    behind()
    for s in range(4):
        order = [0, 1] if s % 2 == 0 else [1, 0]
        for l in range(layers):
            p.extend_step([ids[i] for i in order], [new] * 2, torch.cat([steps[s * layers + l][i] for i in order]), q, o, lse)
        got.append([held(p, r, n + new, layers) for r in ids])
        p.truncate(ids, [n] * 2)
    for s, pair in enumerate(got):
        for i, x in enumerate(pair):
            want = torch.cat([rows[i], torch.stack([steps[s * layers + l][i] for l in range(layers)])], 1)
            assert torch.equal(x, want), (s, i)
    for r in ids:
        p.close(r)
    p.destroy()


@pytest.mark.parametrize("call", ["keep", "evict"])
def test_pages_that_wait_in_a_device_stack_make_room(call):
    """A stack that holds all that open requests may still take gives pages back for those
    that take the place of shared ones."""
    print(f"[case] a full stack, {call}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(4)
    chunk = 16 * P * 2 * ROW  # sixteen pages are the budget
    p = cpl.Pool(page_tokens=P, pool_bytes=chunk, chunk_bytes=chunk, device=0, device_pages=1)
    m = p.register(**GEOMS[NAME])
    a, b, c = p.open(m, 4 * P), p.open(m, 4 * P), p.open(m, 8 * P)
    rows, more = normal(gen, 2 * P, ROW), normal(gen, P + 1, ROW)
    p.append([a], [2 * P], rows)
    p.fork([a], [b])
    p.append([c], [P], more[:P].contiguous())
    q = normal(gen, 1, HQ, DK)
    o, lse = torch.zeros(1, HQ, DV, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, HQ, device="cuda")
    p.decode_step([c], [1], more[P:].contiguous(), q, o, lse)  # takes its page on the device
    places = [[1, 3, 5, 6, 7], [0, 2, 3, 4, 7]]
    if call == "keep":
        p.keep([a, b], [0, 0], [5, 5], sum(places, []))
    else:
        w = [torch.tensor([[float(t in x) for t in range(2 * P)]] * HKV, device="cuda") for x in places]
        p.evict([a, b], [5, 5], w)
    s = p.stats()
    assert (s["pages_used"], s["pages_reserved"]) == (6, 16)
    assert torch.equal(held(p, a, 5)[0], rows[places[0]]) and torch.equal(held(p, b, 5)[0], rows[places[1]])
    assert torch.equal(held(p, c, P + 1)[0], more)
    fill = [normal(gen, k, ROW) for k in (4 * P - 5, 4 * P - 5, 7 * P - 1)]
    p.append([a, b, c], [len(x) for x in fill], torch.cat(fill))
    assert torch.equal(held(p, a, 4 * P)[0], torch.cat([rows[places[0]], fill[0]]))
    assert torch.equal(held(p, c, 8 * P)[0], torch.cat([more, fill[2]]))
    for r in (a, b, c):
        p.close(r)
    assert p.stats()["pages_used"] == p.stats()["pages_reserved"] == 0
    p.destroy()


def test_entries_go_round_their_memory():
    """Appends of 1,000 entries each, dropped and placed again in another order, with no
    waiting in between: more of them than the memory that they are copied from holds."""
    print("[case] entries round and round", flush=True)
    layers, n, rounds = 2, 2000, 160
    gen = torch.Generator(device="cuda").manual_seed(5)
    chunk = 16 * P * 2 * ROW
    p = cpl.Pool(page_tokens=P, pool_bytes=300 * chunk, chunk_bytes=chunk, device=0)
    m = p.register(**GEOMS[NAME], n_layers=layers)
    ids = [p.open(m, n) for _ in range(2)]
    rows = [normal(gen, layers, n, ROW) for _ in range(3)]
    wrong = torch.zeros(rounds, 2, dtype=torch.int64, device="cuda")
    out = torch.zeros(layers, n, ROW, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    behind()
    for i in range(rounds):
        for k in ((0, 1), (1, 0))[i % 2]:
            p.append([ids[k]], [n], rows[(i + k) % 3])
        for k in range(2):
            p.gather(ids[k], 0, n, out)
            wrong[i, k] = (out != rows[(i + k) % 3]).sum()
        p.truncate(ids, [0, 0])
    assert (wrong == 0).all(), wrong.nonzero()
    for r in ids:
        p.close(r)
    p.destroy()
