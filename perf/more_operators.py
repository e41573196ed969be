"""Timing cases of the operators around drafted trees and caches that are cut
down: attention of a tree of drafted tokens over the pool, keeping the tokens
of an accepted path, the weight that queries give to each cached token, and
evicting the tokens of least weight.

A case names what runs (``do``), the model's geometry and its requests. Values
are normal draws made on the GPU from the seed; lengths, trees and accepted
paths come from the case alone.

  tree    cp_tree_build makes the masks and depths of the drafted trees from
          their parents, cp_attn_tree attends: the last tokens of every request
          are its tree, and see the context and their own ancestors.
  draft   a whole speculative step: cp_request_truncate drops what the last
          step left, cp_tree_build, cp_attn_tree_step places the drafted rows,
          keys rotated by depth, and attends, cp_request_keep keeps the path
          that was accepted.
  weights cp_attn_weights: what the last n_q tokens of every request give to
          each cached token, per KV head, added to the decayed sum so far.
  evict   cp_kv_evict keeps the heaviest tokens of every layer and KV head.
          "fork": a branch of a prompt that others go on with is cut down
          (cp_request_fork first); otherwise a prompt is stored and cut
          (cp_kv_append first). cp_kv_gather reads what is left.
"""
from __future__ import annotations

import math
import random

import torch

own = False

CHUNK = 2 << 20
SEG = 64  # elements: every row, page and chunk is a whole number of these

# kind, query heads, KV heads, head width (MLA: latent 512 + rotary 64)
MODELS = {
    "mla16": ("mla", 16, 1, 0),
    "mla128": ("mla", 128, 1, 0),
    "mqa32": ("gqa", 32, 1, 128),
    "gqa32x8": ("gqa", 32, 8, 128),
    "gqa32x4": ("gqa", 32, 4, 128),
    "gqa28x4": ("gqa", 28, 4, 128),
    "gqa24x8": ("gqa", 24, 8, 128),
    "gqa16x4d64": ("gqa", 16, 4, 64),
    "gqa8x8d64": ("gqa", 8, 8, 64),
}


def widths(name):
    """(query heads, KV heads, K width, V width, elements of a logical row)"""
    kind, hq, hkv, d = MODELS[name]
    return (hq, 1, 576, 512, 576) if kind == "mla" else (hq, hkv, d, d, 2 * hkv * d)


def _is_mla(name):
    return MODELS[name][0] == "mla"


def _scale(name):
    return 1 / math.sqrt(192.0 if _is_mla(name) else widths(name)[2])


# ------------------------------------------------------------------- cases

def listed():
    return [
        # smallest: a few drafted tokens of one short request
        dict(name="tree_small", do="tree", model="mla16", lens="300", nodes=8),
        # trees of a serving batch over mixed contexts
        dict(name="tree_batch", do="tree", model="gqa32x8", requests=8, lo=1000, hi=16384, lens_seed=4, nodes=61),
        # a wide tree over a long context, scores falling with distance
        dict(name="tree_slopes", do="tree", model="gqa8x8d64", lens="40000", nodes=129, slopes=True),
        # a speculative step of a small batch: place, attend, keep what was accepted
        dict(name="draft_small", do="draft", model="gqa28x4", requests=4, lo=500, hi=8000, lens_seed=5, nodes=13, rot=128,
             layout="half"),
        # the same with a latent-attention model and wide trees
        dict(name="draft_latent", do="draft", model="mla16", requests=12, lo=1000, hi=16384, lens_seed=6, nodes=64, rot=64,
             layout="interleaved"),
        # single tokens: their weights join the sums of a long decode
        dict(name="weights_token", do="weights", model="gqa32x8", requests=16, lo=512, hi=32768, lens_seed=6, new=1,
             decay=0.98),
        # a prompt's last tokens observe it
        dict(name="weights_window", do="weights", model="gqa32x4", lens="30001", new=32),
        # the largest: every token of prompts is weighed
        dict(name="weights_prompt", do="weights", model="gqa32x8", lens="8192 5000", new=8192),
        # observers of a latent-attention model, the sums so far halved
        dict(name="weights_latent", do="weights", model="mla16", requests=4, lo=2000, hi=16384, lens_seed=7, new=64, decay=0.5),
        # small caches of several layers cut to their budget
        dict(name="evict_layers", do="evict", model="gqa16x4d64", layers=4, requests=6, lo=800, hi=5000, lens_seed=8,
             share=3, first=4, last=64, fork=True),
        # a prompt is stored and cut to an eighth
        dict(name="evict_prompt", do="evict", model="gqa32x8", lens="16384 9001", share=8, first=4, last=32),
        # long prompts of a latent-attention model, kept for others, branch into short ones
        dict(name="evict_fork", do="evict", model="mla16", lens="65536 30000 12345", share=4, first=16, last=128, fork=True),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """One more case of the listed ranges."""
    do = rng.choice(["tree", "tree", "draft", "weights", "weights", "evict", "evict"])
    case = dict(do=do, model=rng.choice(sorted(MODELS)), lens_seed=rng.randrange(1 << 20),
                page_tokens=rng.choice([64, 64, 64, 32, 128]), lo=rng.choice([1, 100, 1000]),
                requests=_log_uniform(rng, 1, 16), hi=_log_uniform(rng, 1000, 65536))
    if do in ("tree", "draft"):
        case["nodes"] = rng.choice([rng.randint(2, 16), _log_uniform(rng, 16, 256)])
        if do == "draft":
            case.update(rot=rng.choice([64, 32]), layout=rng.choice(["half", "interleaved"]))
        mask = rng.choice(["none", "none", "slopes", "window", "cap"])
        if mask == "slopes":
            case["slopes"] = True
        elif mask == "window":
            case["window"] = _log_uniform(rng, 100, 8192)
        elif mask == "cap":
            case["softcap"] = rng.choice([20.0, 50.0])
    elif do == "weights":
        case["new"] = rng.choice([1, rng.randint(2, 16), _log_uniform(rng, 16, 64), _log_uniform(rng, 64, 8192)])
        case["decay"] = rng.choice([0.0, 1.0, 0.9])
        mask = rng.choice(["none", "none", "window", "cap"])
        if mask == "window":
            case["window"] = _log_uniform(rng, 100, 8192)
        elif mask == "cap":
            case["softcap"] = 30.0
    else:
        case.update(layers=rng.choice([1, 1, 2, 5]), share=rng.choice([2, 3, 8]), first=rng.choice([0, 4]),
                    last=rng.choice([0, 16, 100]), fork=rng.random() < 0.6)
    limit = listed()[7]  # "weights_prompt"
    while work(case)["flops"] > work(limit)["flops"] * 0.8 or work(case)["bytes"] > 3e8:  # no more than the largest
        case["requests"] = max(1, case["requests"] // 2)
        case["hi"] = max(case["lo"], case["hi"] * 3 // 4)
        if "new" in case:
            case["new"] = max(1, case["new"] * 3 // 4)
    return case


def _lens(case):
    """Per request (tokens before the call's own, tokens of the call). The
    tokens of a tree or of a weighing call are the last of the context; those of
    a draft come behind it; an eviction has none."""
    if "lens" in case:
        lens = [int(x) for x in case["lens"].split()]
    else:
        rng = random.Random(case["lens_seed"])
        lens = [_log_uniform(rng, case["lo"], max(case["lo"], case["hi"])) for _ in range(case["requests"])]
    if case["do"] == "evict":
        return [(n, 0) for n in lens]
    if case["do"] == "weights":
        return [(n - min(n, case["new"]), min(n, case["new"])) for n in lens]
    rng = random.Random(len(lens))  # trees of about the size asked for
    return [(n, max(1, case["nodes"] - rng.randrange(1 + case["nodes"] // 4))) for n in lens]


def _trees(case):
    """Per request its tree's parents (-1: a child of the context's last token)
    and the accepted path, as indices into the tree."""
    rng = random.Random(case.get("lens_seed", 0) + 17)
    out = []
    for _, n in _lens(case):
        width = rng.randint(1, 12)
        parents = [-1 if t == 0 or rng.random() < 0.1 else rng.randrange(max(0, t - width), t) for t in range(n)]
        node, path = rng.randrange(n) if rng.random() < 0.9 else -1, []
        while node >= 0:
            path.append(node)
            node = parents[node]
        out.append((parents, path[::-1]))
    return out


def _keep(case):
    """Per request the tokens that an eviction keeps."""
    least = case.get("first", 0) + case.get("last", 0)
    return [min(n, max(least, n // case["share"])) for n, _ in _lens(case)]


def _seen(case):
    """Pairs of a query token and a key that it sees, and keys that any sees, per request."""
    out = []
    trees = _trees(case) if case["do"] in ("tree", "draft") else None
    W = case.get("window", 0)
    for i, (base, new) in enumerate(_lens(case)):
        if trees:
            pairs, depth = 0, []
            for p in trees[i][0]:
                depth.append(0 if p < 0 else depth[p] + 1)
                pos = base + depth[-1]
                pairs += base - min(base, max(0, pos - W + 1) if W else 0) + depth[-1] + 1
            out.append((pairs, min(base, base if not W else W) + new))
        else:
            n = base + new
            if W:
                pairs = sum(min(p + 1, W) for p in range(base, n))
                out.append((pairs, min(n, new + W - 1)))
            else:
                out.append((new * base + new * (new + 1) // 2, n))
    return out


def work(case):
    hq, hkv, dk, dv, row = widths(case["model"])
    do, moved, flops = case["do"], 0, 0
    if do == "evict":
        L = case.get("layers", 1)
        for (n, _), k in zip(_lens(case), _keep(case)):
            # the kept rows read and written (a stored prompt: its rows read and
            # written), the sums read, those of kept tokens and their numbers written
            moved += L * (4 * row * k + hkv * (4 * n + 8 * k) + (0 if case.get("fork") else 4 * row * n))
        return {"bytes": moved, "flops": 0}
    for (base, new), (pairs, keys) in zip(_lens(case), _seen(case)):
        if do == "weights":
            moved += 2 * hkv * dk * keys + new * hq * (2 * dk + 4)
            moved += hkv * 4 * (base + new) * (2 if case.get("decay") else 1)
            flops += 2 * dk * hq * pairs
            continue
        moved += 2 * row * keys + new * hq * (2 * dk + 2 * dv + 4) + 4 * new
        flops += 2 * (dk + dv) * hq * pairs
        if do == "draft":  # the new rows: read and written
            moved += 4 * row * new
            flops += 3 * new * case["rot"] * (1 if _is_mla(case["model"]) else hkv)
    if do == "draft":  # rows of accepted paths, where they move
        moved += 4 * row * sum(a != b for _, path in _trees(case) for a, b in enumerate(path))
    return {"bytes": moved, "flops": flops}


# ---------------------------------------------------------------- rotation

def _rotated_rows(rows, case, positions):
    """Logical rows [tokens][row] with their keys turned, in 32 bits (angles in
    64: far positions times frequencies lose the angle in 32)."""
    name = case["model"]
    _, hkv, dk, _, _ = widths(name)
    half = case["rot"] // 2
    f = 10000.0 ** (-2 * torch.arange(half, dtype=torch.float64, device="cuda") / case["rot"])
    ang = positions.double()[:, None] * f
    cos, sin = torch.cos(ang).float()[:, None], torch.sin(ang).float()[:, None]
    y = rows.float()
    part = y[:, None, 512:] if _is_mla(name) else y[:, :hkv * dk].view(-1, hkv, dk)
    part = part[..., :case["rot"]]
    if case["layout"] == "half":
        at = (slice(0, half), slice(half, None))
    else:
        at = (slice(0, None, 2), slice(1, None, 2))
    a, b = part[..., at[0]].clone(), part[..., at[1]].clone()
    part[..., at[0]] = a * cos - b * sin
    part[..., at[1]] = a * sin + b * cos
    return y


# ------------------------------------------------------------------ states

def _segments(name, P, pages, positions):
    """Indices, in units of SEG elements of the pool, of the rows at these
    positions of a request that holds these pages: [tokens][row / SEG]."""
    _, hkv, dk, _, row = widths(name)
    per_chunk = CHUNK // (2 * P * row)
    page = torch.tensor(pages, dtype=torch.int64)[positions // P]
    start = (page // per_chunk) * (CHUNK // 2) + (page % per_chunk) * (P * row)
    slot = (positions % P)[:, None]
    if _is_mla(name):
        at = start[:, None] + slot * row + torch.arange(0, row, SEG)
    else:  # [KV head][K: P rows | V: P rows]
        e = torch.arange(0, row, SEG)
        v, head, off = e // (hkv * dk), e % (hkv * dk) // dk, e % dk
        at = start[:, None] + ((2 * head + v) * P) * dk + slot * dk + off
    return at // SEG


class State:
    """The case's requests with what they hold, and the call's buffers. The
    program holds ids, counts and device addresses ready, as a serving loop
    does."""

    def __init__(self, case, seed):
        self.case, name = case, case["model"]
        self.do = do = case["do"]
        hq, hkv, dk, dv, row = widths(name)
        self.P = P = case.get("page_tokens", 64)
        self.L = L = case.get("layers", 1)
        self.lens = _lens(case)
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, sigma=1.0):
            return torch.empty(*shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, sigma, generator=gen)

        in_place = do in ("tree", "weights")  # the call's tokens are held already
        self.held = [normal(L, b + (n if in_place else 0), row, sigma=math.sqrt(0.5)) for b, n in self.lens]
        self.counts = [n for _, n in self.lens]
        total = sum(self.counts)
        self.slopes = None
        if case.get("slopes"):
            self.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], device="cuda")
        if total:
            self.q = normal(total, hq, dk)
        if do in ("tree", "draft"):
            trees = _trees(case)
            self.out = torch.zeros(total, hq, dv, dtype=torch.bfloat16, device="cuda")
            self.lse = torch.zeros(total, hq, device="cuda")
            self.parents = torch.tensor([p for t, _ in trees for p in t], dtype=torch.int32, device="cuda")
            self.words = -(-max(self.counts) // 32)
            self.mask = torch.zeros(total, self.words, dtype=torch.int32, device="cuda")
            self.depth = torch.zeros(total, dtype=torch.int32, device="cuda")
            self.deepest = 0
            for t, _ in trees:
                d = []
                for p in t:
                    d.append(0 if p < 0 else d[p] + 1)
                self.deepest = max(self.deepest, max(d))
            self.paths = [path for _, path in trees]
        if do == "draft":
            self.rows = normal(total, row, sigma=math.sqrt(0.5))
        if do == "weights":
            self.decay = case.get("decay", 0.0)
            self.old = [torch.rand(hkv, b + n, generator=gen, device="cuda") for b, n in self.lens]
            self.new = [torch.zeros(hkv, b + n, device="cuda") for b, n in self.lens]
            self.lse = _plain_lse(self)  # as the attention of these queries left it
        if do == "evict":
            self.keep = _keep(case)
            # sums of a long run: a few heavy tokens, many light ones, some that nothing looked at
            self.old = [(torch.randn(L, hkv, n, generator=gen, device="cuda") * 2).exp() *
                        (torch.rand(L, hkv, n, generator=gen, device="cuda") > 0.03) for n, _ in self.lens]
            self.new = [torch.zeros_like(w) for w in self.old]
            self.kept = [torch.zeros(L, hkv, k, dtype=torch.int32, device="cuda") for k in self.keep]
            self.left = [torch.zeros(L, k, row, dtype=torch.bfloat16, device="cuda") for k in self.keep]
            self.rows = None if case.get("fork") else torch.cat([h.view(-1, row) for h in self.held])
        # the pages a request holds are the lowest free ones, request by request
        per_chunk = CHUNK // (2 * P * row)
        held = [-(-(b + (n if in_place else 0)) // P) for b, n in self.lens]
        new = [-(-(b + n) // P) - -(-b // P) if do == "draft" else 0 for b, n in self.lens]
        pages = L * (sum(held) * (2 if case.get("fork") else 1) + sum(new) + 2 * len(held))
        self.mem = torch.zeros((-(-pages // per_chunk) + 1) * CHUNK // 2, dtype=torch.bfloat16, device="cuda")
        if not own and do == "draft":
            k, tables = 0, []
            for h in held:
                tables.append(list(range(k, k + h)))
                k += h
            for t, m in zip(tables, new):
                t += range(k, k + m)
                k += m
            segs = self.mem.view(-1, SEG)
            for t, kv in zip(tables, self.held):
                segs[_segments(name, P, t, torch.arange(kv.shape[1])).to("cuda")] = kv[0].view(kv.shape[1], -1, SEG)
            self.new_at = torch.cat([_segments(name, P, t, torch.arange(b, b + n))
                                     for t, (b, n) in zip(tables, self.lens)]).to("cuda")
            first = [0]
            for n in self.counts:
                first.append(first[-1] + n)
            self.path_to = torch.tensor([f + k for f, path in zip(first, self.paths) for k in range(len(path))],
                                        device="cuda", dtype=torch.int64)
            self.path_from = torch.tensor([f + t for f, path in zip(first, self.paths) for t in path], device="cuda",
                                          dtype=torch.int64)
        if do == "draft":
            self.bases = torch.cat([torch.full((n,), b) for b, n in self.lens]).to("cuda", torch.int32)
        if own:
            self._open(name)
        torch.cuda.synchronize()

    def _open(self, name):
        from paper_2606_24506_amd import crosspool as cpl

        case, do = self.case, self.do
        kind, hq, hkv, d = MODELS[name]
        self.device = torch.cuda.current_device()
        self.pool = cpl.Pool(page_tokens=self.P, pool_bytes=2 * self.mem.numel(), chunk_bytes=CHUNK, device=self.device,
                             device_mem=self.mem.data_ptr())
        if kind == "mla":
            m = self.pool.register(cpl.CP_KIND_MLA, hq, 1, latent_dim=512, rope_dim=64, softmax_scale=_scale(name),
                                   n_layers=self.L)
        else:
            m = self.pool.register(cpl.CP_KIND_GQA, hq, hkv, head_dim=d, n_layers=self.L)
        self.stream = torch.cuda.current_stream().cuda_stream
        self.all_ids = held = [self.pool.open(m, b + n) for b, n in self.lens]
        if do != "evict" or case.get("fork"):
            for rid, kv in zip(held, self.held):
                if kv.shape[1]:
                    self.pool.append([rid], [kv.shape[1]], kv, self.stream)
        ids = held
        if do == "evict" and case.get("fork"):
            ids = [self.pool.open(m, b) for b, _ in self.lens]
            self.all_ids = held + ids
            self.parents_of = cpl.i32_array(held)
        self.ids = cpl.i32_array(ids)
        self.n_new = cpl.i32_array(self.counts)
        self.opts = dict(softcap=case.get("softcap", 0.0), window=case.get("window", 0))
        if self.slopes is not None:
            self.opts["slopes"] = self.slopes
        if do == "draft":
            self.drop = cpl.i64_array([b for b, _ in self.lens])
            self.rope = cpl.Rope(case["rot"], device=self.device, layout=case["layout"])
            self.n_path = cpl.i32_array([len(p) for p in self.paths])
            self.path = cpl.i32_array([t for p in self.paths for t in p])
        if do in ("weights", "evict"):
            self.w_old = cpl.token_rows(self.old) if do == "evict" or self.decay else None
            self.w_new = cpl.token_rows(self.new)
        if do == "evict":
            self.n_keep = cpl.i64_array(self.keep)
            self.w_kept = cpl.token_rows(self.kept)
            self.zero = cpl.i64_array([0] * len(ids))
            self.n_held = cpl.i32_array([n for n, _ in self.lens])
            self.gathers = list(zip(ids, self.keep, self.left))

    def __del__(self):
        pool = getattr(self, "pool", None)
        if pool is None:
            return
        torch.cuda.synchronize()
        for r in getattr(self, "all_ids", []):
            pool.close(r)
        pool.destroy()


def prepare(case, seed):
    return State(case, seed)


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    if s.do == "weights":
        s.pool.weights(s.ids, s.n_new, s.q, s.lse, s.w_new, s.stream, old=s.w_old, decay=s.decay, **s.opts)
        return s.new
    if s.do == "evict":
        s.pool.truncate(s.ids, s.zero, s.stream)
        if s.case.get("fork"):
            s.pool.fork(s.parents_of, s.ids, None, s.stream)
        else:
            s.pool.append(s.ids, s.n_held, s.rows, s.stream)
        s.pool.evict(s.ids, s.n_keep, s.w_old, s.stream, new=s.w_new, kept=s.w_kept, first=s.case.get("first", 0),
                     last=s.case.get("last", 0))
        for rid, k, left in s.gathers:
            s.pool.gather(rid, 0, k, left, s.stream)
        return s.left, s.kept, s.new
    from paper_2606_24506_amd import crosspool as cpl

    if s.do == "draft":
        s.pool.truncate(s.ids, s.drop, s.stream)
    cpl.cp_tree_build(s.n_new, s.parents, s.mask, s.depth, s.stream)
    if s.do == "tree":
        s.pool.tree(s.ids, s.n_new, s.q, s.out, s.lse, s.mask, s.depth, s.stream, **s.opts)
        return s.out, s.lse, s.depth
    s.pool.tree_step(s.ids, s.n_new, s.rows, s.q, s.out, s.lse, s.mask, s.depth, s.stream, rope=s.rope, **s.opts)
    s.pool.keep(s.ids, s.drop, s.n_path, s.path, s.stream)
    return s.out, s.lse, s.depth, s.mem


# -------------------------------------------------------------- plain form

def _run_plain(s):
    if s.do == "weights":
        return _plain_weights(s)
    if s.do == "evict":
        return _plain_evict(s)
    # ancestors, walking up from every token at once
    total = s.parents.shape[0]
    at = torch.arange(total, device="cuda")
    first = torch.cat([torch.full((n,), sum(s.counts[:i])) for i, n in enumerate(s.counts)]).to("cuda")
    sees = torch.zeros(total, max(s.counts) + 1, dtype=torch.bool, device="cuda")
    node, depth = at - first, torch.full_like(s.depth, -1)
    for _ in range(s.deepest + 1):
        real = node >= 0
        sees[at, torch.where(real, node, sees.shape[1] - 1)] = True
        depth += real.int()
        up = s.parents[(first + node.clamp(min=0))].long()
        node = torch.where(real, up, -1)
    if s.do == "tree":
        return (*_plain_attention(s, sees, depth, None), depth)
    rows = _rotated_rows(s.rows, s.case, s.bases + depth).to(torch.bfloat16)
    got = _plain_attention(s, sees, depth, rows)
    segs = s.mem.view(-1, SEG)
    segs[s.new_at] = rows.view(rows.shape[0], -1, SEG)
    segs[s.new_at[s.path_to]] = segs[s.new_at[s.path_from]]
    return (*got, depth, s.mem)


def _scores(s, q, k, heads, far):
    """Scores [tokens][g][keys] in 32 bits of queries [tokens][g][K width] and keys [n][K width]."""
    t, g, dk = q.shape
    x = (q.reshape(-1, dk).float() @ k.float().t().contiguous()).view(t, g, -1) * _scale(s.case["model"])
    if s.case.get("softcap"):
        x = torch.tanh(x / s.case["softcap"]) * s.case["softcap"]
    if s.slopes is not None:
        x = x - s.slopes[heads][None, :, None] * far[:, None, :]
    return x


def _plain_attention(s, sees, depth, rows):
    name = s.case["model"]
    hq, hkv, dk, dv, _ = widths(name)
    g = hq // hkv
    W = s.case.get("window", 0)
    out, lse = torch.empty_like(s.out), torch.empty_like(s.lse)
    at = 0
    for i, (base, new) in enumerate(s.lens):
        kv = s.held[i][0] if rows is None else torch.cat([s.held[i][0], rows[at:at + new]])
        j = torch.cat([torch.arange(base, device="cuda"), base + depth[at:at + new].long()])  # where each key stands
        p = base + depth[at:at + new].long()[:, None]
        see = torch.cat([(j[None, :base] > p - W) if W else torch.ones(new, base, dtype=torch.bool, device="cuda"),
                         sees[at:at + new, :new]], dim=1)
        far = (p - j[None]).abs().float()
        for h in range(hkv):
            heads = slice(h * g, (h + 1) * g)
            k = kv if _is_mla(name) else kv[:, h * dk:(h + 1) * dk]
            v = kv[:, :dv] if _is_mla(name) else kv[:, (hkv + h) * dv:(hkv + h + 1) * dv]
            x = _scores(s, s.q[at:at + new, heads], k, heads, far).masked_fill(~see[:, None, :], -math.inf)
            m = x.amax(dim=2, keepdim=True)
            e = torch.exp(x - m)
            z = e.sum(dim=2, keepdim=True)
            out[at:at + new, heads] = ((e.view(new * g, -1) @ v.float()).view(new, g, dv) / z).to(out.dtype)
            lse[at:at + new, heads] = (m + torch.log(z))[..., 0]
        at += new
    return out, lse


def _blocks(s):
    """Of every request, KV head and block of query tokens: (request, its place
    in the call, head, query heads, tokens of the call, scores with what is not seen at -inf)."""
    name = s.case["model"]
    hq, hkv, dk, _, _ = widths(name)
    g = hq // hkv
    W = s.case.get("window", 0)
    at = 0
    for i, (base, new) in enumerate(s.lens):
        n = base + new
        step = max(1, (1 << 28) // (g * n))  # query tokens at once, for memory's sake
        j = torch.arange(n, device="cuda")[None]
        for a in range(0, new, step):
            b = min(new, a + step)
            p = torch.arange(base + a, base + b, device="cuda")[:, None]
            hide = (j > p) | (j <= p - W) if W else j > p
            for h in range(hkv):
                heads = slice(h * g, (h + 1) * g)
                k = s.held[i][0]
                k = k if _is_mla(name) else k[:, h * dk:(h + 1) * dk]
                x = _scores(s, s.q[at + a:at + b, heads], k, heads, None)
                yield i, h, heads, slice(at + a, at + b), x.masked_fill_(hide[:, None, :], -math.inf)
        at += new


def _plain_lse(s):
    lse = torch.empty(s.q.shape[0], s.q.shape[1], device="cuda")
    for _, _, heads, toks, x in _blocks(s):
        m = x.amax(dim=2)
        lse[toks, heads] = m + torch.log(torch.exp(x.sub_(m[..., None])).sum(dim=2))
    return lse


def _plain_weights(s):
    new = [w * s.decay if s.decay else torch.zeros_like(w) for w in s.old]
    for i, h, heads, toks, x in _blocks(s):
        new[i][h] += torch.exp(x.sub_(s.lse[toks, heads][..., None])).sum(dim=(0, 1))
    return new


def _plain_evict(s):
    _, hkv, _, _, row = widths(s.case["model"])
    F, R = s.case.get("first", 0), s.case.get("last", 0)
    lefts, kepts, news = [], [], []
    for kv, w, keep in zip(s.held, s.old, s.keep):
        if not s.case.get("fork"):
            kv = kv.clone()  # the prompt is stored
        L, n = kv.shape[:2]
        rank = w.clone()
        rank[..., :F] = math.inf
        rank[..., n - R:] = math.inf
        order = torch.sort(rank, dim=-1, descending=True, stable=True)[1][..., :keep]
        kept = torch.sort(order, dim=-1)[0]  # [L][KV heads][keep]
        new = torch.zeros_like(w)
        new[..., :keep] = torch.gather(w, 2, kept)
        parts = kv.view(L, n, 1, 1, row) if hkv == 1 and _is_mla(s.case["model"]) else kv.view(L, n, 2, hkv, -1)
        idx = kept.permute(0, 2, 1)[:, :, None, :, None].expand(L, keep, parts.shape[2], hkv, parts.shape[4])
        lefts.append(torch.gather(parts, 1, idx).reshape(L, keep, row))
        kepts.append(kept.int())
        news.append(new)
    return lefts, kepts, news


# ---------------------------------------------------------- 64-bit results

def exact(case, seed):
    s = prepare(case, seed)
    if case["do"] == "weights":
        return _weights64(s)
    if case["do"] == "evict":
        return _evict64(s)
    name = case["model"]
    hq, hkv, dk, dv, row = widths(name)
    trees = _trees(case)
    depths = []
    for parents, _ in trees:
        d = []
        for p in parents:
            d.append(0 if p < 0 else d[p] + 1)
        depths.append(d)
    new = rows = None
    if case["do"] == "draft":
        pos = torch.tensor([b + x for (b, _), d in zip(s.lens, depths) for x in d], device="cuda", dtype=torch.float64)
        new = _turn64(s.rows, case, pos)
        rows = new.to(torch.bfloat16)  # what the cache holds
    outs, lses, at = [], [], 0
    for i, (base, n) in enumerate(s.lens):
        kv = s.held[i][0].double()
        if rows is not None:
            kv = torch.cat([kv, rows[at:at + n].double()])
        see = torch.zeros(n, base + n, dtype=torch.bool)
        for t in range(n):
            lo = max(0, base + depths[i][t] - case["window"] + 1) if case.get("window") else 0
            see[t, min(lo, base):base] = True
            a = t
            while a >= 0:
                see[t, base + a] = True
                a = trees[i][0][a]
        see = see.to("cuda")
        stand = torch.tensor(list(range(base)) + [base + x for x in depths[i]], device="cuda", dtype=torch.float64)
        dist = (stand[base:, None] - stand[None]).abs()
        for h in range(hq):
            c = h // (hq // hkv)
            k = kv if _is_mla(name) else kv[:, c * dk:(c + 1) * dk]
            v = kv[:, :dv] if _is_mla(name) else kv[:, (hkv + c) * dv:(hkv + c + 1) * dv]
            x = torch.mm(s.q[at:at + n, h].double(), k.t().contiguous()) * _scale(name)
            if case.get("softcap"):
                x = case["softcap"] * torch.tanh(x / case["softcap"])
            if s.slopes is not None:
                x = x - s.slopes[h].double() * dist
            x = torch.where(see, x, torch.tensor(-math.inf, dtype=torch.float64, device="cuda"))
            z = torch.logsumexp(x, dim=1)
            outs.append(torch.mm(torch.exp(x - z[:, None]), v.contiguous()))
            lses.append(z)
        at += n
    out = torch.cat([torch.stack(outs[i * hq:(i + 1) * hq], 1) for i in range(len(s.lens))])
    lse = torch.cat([torch.stack(lses[i * hq:(i + 1) * hq], 1) for i in range(len(s.lens))])
    depth = torch.tensor([x for d in depths for x in d], dtype=torch.int32, device="cuda")
    if case["do"] == "tree":
        return out, lse, depth
    return out, lse, depth, _mem64(case, s, new, [path for _, path in trees])


def _turn64(rows, case, pos):
    """Rotation as complex products."""
    name = case["model"]
    _, hkv, dk, _, row = widths(name)
    half = case["rot"] // 2
    f = torch.tensor([math.pow(10000.0, -2.0 * i / case["rot"]) for i in range(half)], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones(pos.shape[0], half, dtype=torch.float64, device="cuda"), torch.outer(pos, f))
    y = rows.double()
    for at in ([512] if _is_mla(name) else [h * dk for h in range(hkv)]):
        part = y[:, at:at + 2 * half].clone()
        if case["layout"] == "half":
            z = torch.complex(part[:, :half].contiguous(), part[:, half:].contiguous()) * turn
            y[:, at:at + 2 * half] = torch.cat([z.real, z.imag], dim=-1)
        else:
            z = torch.view_as_complex(part.view(-1, half, 2)) * turn
            y[:, at:at + 2 * half] = torch.view_as_real(z).flatten(-2)
    return y


def _mem64(case, s, new, paths):
    """The pool's memory after the step: the held rows, behind them the drafted
    ones (each request's next page the lowest free one), of which the accepted
    path's take the first places."""
    name, P = case["model"], s.P
    _, hkv, dk, _, row = widths(name)
    per_chunk = CHUNK // (2 * P * row)
    mem = torch.zeros(s.mem.numel(), dtype=torch.float64, device="cuda")
    free, tables, at = 0, [], 0
    for base, _ in s.lens:
        k = (base + P - 1) // P
        tables.append([free + i for i in range(k)])
        free += k
    for i, (base, n) in enumerate(s.lens):
        mine = new[at:at + n].clone()
        at += n
        for k, t in enumerate(paths[i]):  # ascending: a row is read before its place is taken
            mine[k] = mine[t].clone()
        whole = torch.cat([s.held[i][0].double(), mine])
        while len(tables[i]) * P < base + n:
            tables[i].append(free)
            free += 1
        for k, page in enumerate(tables[i]):
            r = whole[k * P:(k + 1) * P]
            start = page // per_chunk * (CHUNK // 2) + page % per_chunk * P * row
            block = mem[start:start + P * row]
            if _is_mla(name):
                block[:r.numel()] = r.reshape(-1)
            else:
                block.view(hkv, 2, P, dk)[:, :, :r.shape[0]] = r.view(-1, 2, hkv, dk).permute(2, 1, 0, 3)
    return mem


def _weights64(s):
    case, name = s.case, s.case["model"]
    hq, hkv, dk, _, _ = widths(name)
    got, at = [], 0
    for i, (base, new) in enumerate(s.lens):
        n = base + new
        sums = s.old[i].double() * s.decay if s.decay else torch.zeros(hkv, n, dtype=torch.float64, device="cuda")
        j = torch.arange(n, device="cuda")
        for h in range(hq):
            c = h // (hq // hkv)
            k = s.held[i][0].double()
            k = (k if _is_mla(name) else k[:, c * dk:(c + 1) * dk]).t().contiguous()
            for a in range(0, new, 4096):
                b = min(new, a + 4096)
                p = torch.arange(base + a, base + b, device="cuda")[:, None]
                x = torch.mm(s.q[at + a:at + b, h].double(), k) * _scale(name)
                if case.get("softcap"):
                    x = case["softcap"] * torch.tanh(x / case["softcap"])
                e = torch.exp(x - s.lse[at + a:at + b, h].double()[:, None])
                e = e * (j[None] <= p)
                if case.get("window"):
                    e = e * (p - j[None] < case["window"])
                sums[c] += e.sum(0)
        at += new
        got.append(sums)
    return got


def _evict64(s):
    """Each layer and head by itself: which tokens stay, their rows and their sums."""
    case, name = s.case, s.case["model"]
    _, hkv, dk, _, row = widths(name)
    first, last = case.get("first", 0), case.get("last", 0)
    lefts, kepts, news = [], [], []
    for kv, w, keep in zip(s.held, s.old, s.keep):
        L, n, _ = kv.shape
        left = torch.zeros(L, keep, row, dtype=torch.float64, device="cuda")
        kept = torch.zeros(L, hkv, keep, dtype=torch.int32, device="cuda")
        new = torch.zeros(L, hkv, n, dtype=torch.float64, device="cuda")
        for l in range(L):
            for h in range(hkv):
                mine = w[l, h].tolist()
                middle = sorted(range(first, max(first, n - last)), key=lambda t: (-mine[t], t))
                sure = set(range(min(first, n))) | set(range(max(0, n - last), n))
                chosen = torch.tensor(sorted(sure | set(middle[:keep - len(sure)])), dtype=torch.int64, device="cuda")
                kept[l, h] = chosen.int()
                new[l, h, :keep] = w[l, h][chosen].double()
                if _is_mla(name):
                    left[l] = kv[l][chosen].double()
                else:
                    for part in (h, hkv + h):
                        left[l, :, part * dk:(part + 1) * dk] = kv[l][chosen][:, part * dk:(part + 1) * dk].double()
        lefts.append(left)
        kepts.append(kept)
        news.append(new)
    return lefts, kepts, news
