"""Forks and truncations while pages wait in the device stacks and entries popped on
the GPU have not been read back: a tight pool with device page stacks runs the same
calls as one without, and both hold the rows that they should."""
import random

import pytest
import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, bits, shape

pytestmark = pytest.mark.gpu

NAME, P, PAGES_PER_CHUNK = "gqa6x2d64", 4, 8


class Twin:
    """The same calls on a pool without and on one with device page stacks."""

    def __init__(self, chunks, layers, seed, models=1):
        self.hq, self.hkv, self.dk, self.dv, self.row, _ = shape(NAME)
        chunk = PAGES_PER_CHUNK * P * 2 * self.row
        self.L = layers
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.pools = [cpl.Pool(page_tokens=P, pool_bytes=chunks * chunk, chunk_bytes=chunk, placement_seed=seed, device=0,
                               device_pages=d) for d in (0, 1)]
        for p in self.pools:
            self.models = [p.register(**GEOMS[NAME], n_layers=layers) for _ in range(models)]
        self.rows = {}  # request -> [layers][tokens][row]
        self.cap, self.of = {}, {}

    def normal(self, *size):
        return torch.empty(*size, dtype=torch.bfloat16, device="cuda").normal_(generator=self.gen)

    def both(self, fn):
        """Runs fn(pool) on both; the statuses, which must agree."""
        got = []
        for p in self.pools:
            try:
                got.append((cpl.CP_OK, fn(p)))
            except cpl.CrossPoolError as e:
                assert e.status in (cpl.CP_ENOSPC, cpl.CP_EINVAL), e
                got.append((e.status, None))
        assert got[0] == got[1], got
        return got[0]

    def open(self, cap, model=0):
        rc, r = self.both(lambda p: p.open(self.models[model], cap))
        if rc == cpl.CP_OK:
            self.rows[r], self.cap[r], self.of[r] = self.normal(self.L, 0, self.row), cap, model
            return r

    def append(self, ids, n_new):
        new = [self.normal(self.L, n, self.row) for n in n_new]
        flat = torch.cat([x.reshape(-1) for x in new] + [self.normal(8)])
        rc, _ = self.both(lambda p: p.append(ids, n_new, flat))
        if rc == cpl.CP_OK:
            for r, x in zip(ids, new):
                self.rows[r] = torch.cat([self.rows[r], x], 1)

    def step(self, ids, how):
        """A token for each request through every layer; no waiting in between."""
        ids = [r for r in ids if self.rows[r].shape[1] < self.cap[r]]
        if not ids:
            return
        n, L = len(ids), self.L
        new = self.normal(n, L, self.row)
        q = self.normal(n, L, self.hq, self.dk)
        outs = []
        for p in self.pools:
            out = torch.zeros(n, L, self.hq, self.dv, dtype=torch.bfloat16, device="cuda")
            lse = torch.zeros(n, L, self.hq, device="cuda")
            if how == "layers":
                p.decode_layers(ids, [1] * n, new, q, out, lse)
            else:
                for l in range(L):
                    o, e = torch.zeros_like(out[:, l].contiguous()), torch.zeros_like(lse[:, l].contiguous())
                    call = p.decode_step if how == "decode" else p.extend_step
                    call(ids, [1] * n, new[:, l].contiguous(), q[:, l].contiguous(), o, e)
                    out[:, l], lse[:, l] = o, e
            outs.append((out, lse))
        assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
        for i, r in enumerate(ids):
            self.rows[r] = torch.cat([self.rows[r], new[i][:, None]], 1)

    def fork(self, src, dst, n_tok):
        rc, _ = self.both(lambda p: p.fork(src, dst, n_tok))
        assert rc == cpl.CP_OK
        for s, d, n in zip(src, dst, n_tok):
            self.rows[d] = self.rows[s][:, :n]

    def truncate(self, ids, to):
        rc, _ = self.both(lambda p: p.truncate(ids, to))
        if rc == cpl.CP_OK:
            for r, n in zip(ids, to):
                self.rows[r] = self.rows[r][:, :n]

    def close(self, r):
        torch.cuda.synchronize()
        self.both(lambda p: p.close(r))
        del self.rows[r], self.cap[r], self.of[r]

    def check(self):
        a, b = (p.stats() for p in self.pools)
        assert (a["pages_used"], a["pages_reserved"]) == (b["pages_used"], b["pages_reserved"])
        for r, want in self.rows.items():
            n = want.shape[1]
            for p in self.pools:
                assert p.ctx_len(r) == n
                got = torch.zeros(self.L, n, self.row, dtype=torch.bfloat16, device="cuda")
                if n:
                    p.gather(r, 0, n, got)
                assert (bits(got) == bits(want)).all(), r

    def end(self):
        for r in list(self.rows):
            self.close(r)
        for p in self.pools:
            s = p.stats()
            assert s["pages_used"] == s["pages_reserved"] == s["chunks_used"] == 0, s
            p.destroy()


@pytest.mark.parametrize("layers", [1, 3])
@pytest.mark.parametrize("how", ["decode", "layers", "extend"])
def test_a_tight_pool_with_waiting_pages(layers, how):
    """The budget is what the requests may take, to the page: the stack holds the
    rest of it when the fork, the truncation and the appends need pages."""
    print(f"[case] device pages {layers} {how}", flush=True)
    # three requests of 16, 16 and 32 tokens: 16 pages a plane
    t = Twin(chunks=2 * layers, layers=layers, seed=5)
    a, b, c = t.open(16), t.open(16), t.open(32)
    assert t.open(1) is None
    t.append([a], [7])
    t.step([a], how)
    t.step([a], how)  # opens a page: popped, and pending until read back
    t.fork([a, a], [b, c], [9, 8])  # shares two whole pages and copies one
    t.step([a, b, c], how)
    t.check()
    t.truncate([b], [3])  # inside a shared page
    t.step([a, b], how)
    t.append([c], [9])
    t.step([a, b, c], how)
    t.check()
    d = t.open(4)  # what the sharing gave back
    t.truncate([a, b, c], [5, 2, 6])  # two more copies, if the place is still there
    t.check()
    for _ in range(20):
        t.step([a, b, c], how)
    t.check()
    t.close(a)
    t.step([b, c], how)
    for r in (b, c):
        t.append([r], [t.cap[r] - t.rows[r].shape[1]])
    t.check()
    if d is not None:
        t.append([d], [4])
    t.check()
    t.end()


@pytest.mark.parametrize("models", [1, 2])
@pytest.mark.parametrize("seed", range(6))
def test_random_calls_of_both_kinds_of_pool(seed, models):
    print(f"[case] device pages random {seed} {models}", flush=True)
    rng = random.Random(seed)
    t = Twin(chunks=24, layers=1 + seed % 3, seed=seed + 1, models=models)
    for k in range(160):
        ids = list(t.rows)
        do = rng.choice(["open", "append", "step", "step", "step", "fork", "truncate", "truncate", "close"])
        if do == "open":
            t.open(rng.randint(1, 60), rng.randrange(models))
        elif do == "append" and ids:
            r = rng.choice(ids)
            t.append([r], [rng.randint(0, 9)])
        elif do == "step" and ids:
            how = rng.choice(["decode", "layers", "extend"])
            some = [r for r in ids if how != "extend" or t.of[r] == t.of[ids[0]]]
            t.step(rng.sample(some, rng.randint(1, min(4, len(some)))), how)
        elif do == "fork" and len(ids) > 1:
            s = rng.choice(ids)
            dst = [r for r in ids if r != s and t.of[r] == t.of[s] and t.rows[r].shape[1] == 0][:2]
            if dst:
                t.fork([s] * len(dst), dst, [rng.randint(0, min(t.rows[s].shape[1], t.cap[r])) for r in dst])
        elif do == "truncate" and ids:
            some = rng.sample(ids, min(len(ids), rng.randint(1, 3)))
            t.truncate(some, [rng.randint(0, t.rows[r].shape[1]) for r in some])
        elif do == "close" and len(ids) > 4:
            t.close(rng.choice(ids))
        if k % 8 == 7:
            t.check()
    for r in list(t.rows):  # an admitted request can always fill its reservation
        t.append([r], [t.cap[r] - t.rows[r].shape[1]])
        assert t.rows[r].shape[1] == t.cap[r]
    t.check()
    t.end()
