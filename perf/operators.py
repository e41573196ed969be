"""Timing cases of the operators around a prompt and its branches: rotary
positions, attention of token chunks and single tokens with capped scores,
distance bias, windows, document and prefix masks, and forking and
truncating requests whose KV lives in the pool.

A case names what runs (``do``), the model's geometry, its requests and the
options of the call. Values are normal draws made on the GPU from the seed;
lengths come from the case alone.

  rope    cp_rope_apply of every query and key head of a batch of tokens.
  append  cp_kv_append_rope of a chunk of prompt rows to every request, behind
          what the request holds (cp_request_truncate puts it back first, as a
          program does that runs a prompt's tail again).
  extend  cp_attn_extend over a loaded batch: the last n_q tokens of every
          request attend over its context.
  step    a speculative step: cp_request_truncate drops the tokens that were
          not accepted, cp_rope_apply rotates the queries, cp_attn_extend_step
          places the drafted tokens' rows, keys rotated, and attends.
  branch  the same step for branches of shared prompts: cp_request_truncate
          empties the branches, cp_request_fork makes them share their parents'
          pages, and each branch goes on with tokens of its own.
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
        # smallest: the queries and keys of four requests' next tokens
        dict(name="rope_token", do="rope", tokens=4, heads="32 8", width=128, rot=128, layout="half", far=4096),
        # a prompt's queries and keys, positions far past the trained context
        dict(name="rope_prompt", do="rope", tokens=8192, heads="32 8", width=128, rot=128, layout="half", far=131072,
             scaling="parts", factor=8.0),
        # the rotary part of a latent-attention model's absorbed queries
        dict(name="rope_latent", do="rope", tokens=5001, heads="16", width=576, offset=512, rot=64,
             layout="interleaved", far=60000, scaling="ntk", factor=4.0),
        # prompt chunks written into the pool, keys rotated on the way
        dict(name="append_rope", do="append", model="gqa24x8", requests=6, lo=500, hi=8000, new=2000, lens_seed=3,
             layout="half", rot=128),
        # single tokens over long caches, scores capped
        dict(name="decode_cap", do="extend", model="gqa32x8", requests=16, lo=512, hi=32768, lens_seed=6, new=1,
             softcap=30.0),
        # one token over a very long cache, scores falling with distance
        dict(name="decode_slope", do="extend", model="gqa8x8d64", lens="262144", new=1, slopes=True),
        # the largest: prompt chunks behind earlier ones, scores capped
        dict(name="prompt_cap", do="extend", model="gqa32x8", lens="16384 9000 4096", new=2048, softcap=50.0),
        # a packed prompt of many documents, none seeing another
        dict(name="prompt_docs", do="extend", model="gqa16x4d64", lens="6001 3333", new=8192, docs=700, lens_seed=5),
        # a prompt chunk of a latent-attention model, in a sliding window
        dict(name="prompt_latent", do="extend", model="mla16", lens="6000 2500", new=1024, window=4096),
        # drafted tokens checked in one step
        dict(name="draft_step", do="step", model="mla16", requests=8, lo=1000, hi=16384, lens_seed=8, new=5,
             layout="interleaved", rot=64),
        # sampled continuations of a few prompts
        dict(name="branches", do="branch", model="gqa24x8", requests=4, lo=500, hi=8000, lens_seed=9, branches=4, new=1,
             layout="half", rot=128),
        # wide beams over one prompt read in both directions
        dict(name="beams", do="branch", model="gqa32x4", lens="3001", branches=16, new=2, prefix=True, layout="half",
             rot=64),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """One more case of the listed ranges."""
    do = rng.choice(["rope", "append", "extend", "extend", "extend", "step", "branch"])
    layout = rng.choice(["half", "interleaved"])
    scaling = rng.choice(["none", "linear", "ntk", "parts"])
    if do == "rope":
        width = rng.choice([64, 128, 256])
        case = dict(do=do, tokens=_log_uniform(rng, 1, 8192), width=width, rot=rng.choice([width, width // 2]),
                    heads=rng.choice(["32 8", "16", "28 4", "8 8", "1"]), far=_log_uniform(rng, 100, 1 << 20))
    else:
        name = rng.choice(sorted(MODELS))
        case = dict(do=do, model=name, lens_seed=rng.randrange(1 << 20), page_tokens=rng.choice([64, 64, 64, 32, 128]),
                    lo=rng.choice([1, 100, 1000]), rot=rng.choice([64, 32]) if do != "extend" else 64)
        case["hi"] = _log_uniform(rng, 1000, 32768)
        case["requests"] = _log_uniform(rng, 1, 32)
        if do == "append":
            case["new"] = _log_uniform(rng, 10, 4000)
        elif do == "extend":
            case["new"] = rng.choice([1, 1, rng.randint(2, 16), _log_uniform(rng, 16, 4096)])
        else:
            case["new"] = rng.choice([1, rng.randint(2, 8)])
        if do == "branch":
            case["branches"] = rng.randint(2, 8)
            case["requests"] = min(8, case["requests"])
        if do != "append":
            mask = rng.choice(["none", "cap", "slopes", "window", "docs", "prefix"])
            if mask == "cap":
                case["softcap"] = rng.choice([20.0, 30.0, 50.0])
            elif mask == "slopes":
                case["slopes"] = True
            elif mask == "window":
                case["window"] = _log_uniform(rng, 100, 4096)
            elif mask == "docs":
                case["docs"] = _log_uniform(rng, 50, 2000)
            elif mask == "prefix":
                case["prefix"] = True
    if do != "extend":
        case["layout"] = layout
        if scaling != "none":
            case.update(scaling=scaling, factor=rng.choice([2.0, 4.0, 8.0]))
    most = work(listed()[6])["flops"] * 0.5  # "prompt_cap"
    while do != "rope" and (work(case)["flops"] > most or work(case)["bytes"] > 4e8):  # no more than the largest case
        case["requests"] = max(1, case["requests"] // 2)
        case["hi"] = max(case["lo"], case["hi"] * 3 // 4)
        case["new"] = max(1, case["new"] * 3 // 4)
    return case


def _lens(case):
    """Per request (tokens held before the call, tokens of the call): an
    extend's are the last of the context, the others' come behind it."""
    if "lens" in case:
        lens = [int(x) for x in case["lens"].split()]
    else:
        rng = random.Random(case["lens_seed"])
        lens = [_log_uniform(rng, case["lo"], max(case["lo"], case["hi"])) for _ in range(case["requests"])]
    if case["do"] == "extend":
        return [(n - min(n, case["new"]), min(n, case["new"])) for n in lens]
    rng = random.Random(len(lens))
    if case["do"] == "append":  # ragged chunks
        return [(n, max(1, case["new"] - rng.randrange(1 + case["new"] // 2))) for n in lens]
    return [(n, case["new"]) for n in lens]


def _spans(case):
    """Per request the first and one past the last visible key of each of its
    query tokens (two lists), before positions are known to any code below."""
    rng = random.Random(case.get("lens_seed", 0) + 1)
    spans = []
    for base, new in _lens(case):
        n = base + new
        starts = [0] * n
        if "docs" in case:
            at = 0
            while at < n:
                end = min(n, at + _log_uniform(rng, max(1, case["docs"] // 8), case["docs"] * 2))
                starts[at:end] = [at] * (end - at)
                at = end
        prefix = _prefix(case, base, new)
        lo, hi = [], []
        for p in range(base, n):
            first = starts[p]
            if case.get("window"):
                first = max(first, p - case["window"] + 1)
            lo.append(first)
            hi.append(max(p + 1, prefix))
        spans.append((lo, hi, starts[base:]))
    return spans


def _prefix(case, base, new):
    """Tokens at the start that see each other: the prompt held before the
    call, or half of a context that the call's tokens end."""
    if not case.get("prefix"):
        return 0
    return (base + new) // 2 if case["do"] == "extend" else base


def work(case):
    if case["do"] == "rope":
        heads = sum(int(h) for h in case["heads"].split())
        elems = case["tokens"] * heads * (case["rot"] if case.get("offset") else case["width"])
        return {"bytes": 4 * elems + 4 * case["tokens"], "flops": 3 * case["tokens"] * heads * case["rot"]}
    hq, hkv, dk, dv, row = widths(case["model"])
    rows = sum(new for _, new in _lens(case))
    k_heads = 1 if _is_mla(case["model"]) else hkv
    if case["do"] == "append":
        return {"bytes": 4 * rows * row, "flops": 3 * rows * k_heads * case["rot"]}
    per = case.get("branches", 1)  # branches share their prompt's rows
    moved = flops = 0
    P = case.get("page_tokens", 64)
    for (base, new), (lo, hi, _) in zip(_lens(case), _spans(case)):
        pairs = sum(b - a for a, b in zip(lo, hi))
        seen = max(hi) - min(lo)
        moved += 2 * row * max(0, seen - (new if case["do"] != "extend" else 0))
        moved += per * new * hq * (2 * dk + 2 * dv + 4)
        flops += per * 2 * (dk + dv) * hq * pairs
        if case["do"] != "extend":  # the new rows: read and written; the queries rotated before
            moved += per * new * (4 * row + 4 * hq * dk)
            flops += per * 3 * new * case["rot"] * (hq + k_heads)
        if case["do"] == "branch":  # a page that the prompt ends in is copied, entries of the others
            moved += per * (4 * row * (base % P) + 8 * (base // P))
    return {"bytes": moved, "flops": flops}


# ---------------------------------------------------------------- rotation

def _rope_desc(case):
    return dict(rot_dim=case["rot"], layout=case["layout"], base=10000.0, scaling=case.get("scaling", "none"),
                factor=case.get("factor", 1.0), orig_len=8192, low_turns=1.0, high_turns=32.0,
                magnitude=0.1 * math.log(case["factor"]) + 1 if case.get("scaling") == "parts" else 1.0)


def _angles(case, positions):
    """Angles [tokens][rot / 2] in 64 bits (far positions times frequencies
    lose the angle in 32) and the factor of sine and cosine."""
    d = _rope_desc(case)
    half = d["rot_dim"] // 2
    i = torch.arange(half, dtype=torch.float64, device=positions.device)
    base = d["base"]
    if d["scaling"] == "ntk":
        base *= d["factor"] ** (d["rot_dim"] / (d["rot_dim"] - 2))
    f = base ** (-2 * i / d["rot_dim"])
    if d["scaling"] == "linear":
        f = f / d["factor"]
    elif d["scaling"] == "parts":
        turns = d["orig_len"] * f / (2 * math.pi)
        keep = ((turns - d["low_turns"]) / (d["high_turns"] - d["low_turns"])).clamp(0, 1)
        f = f * keep + f / d["factor"] * (1 - keep)
    return positions.double()[:, None] * f, d["magnitude"]


def _rotated(x, case, positions, offset, real):
    """x [tokens][heads][width] with its rotary part turned, in type real."""
    ang, mag = _angles(case, positions)
    cos, sin = (torch.cos(ang) * mag).to(real)[:, None], (torch.sin(ang) * mag).to(real)[:, None]
    y = x.to(real, copy=True)
    part = y[..., offset:offset + case["rot"]]
    if case["layout"] == "half":
        h = case["rot"] // 2
        a, b = part[..., :h].clone(), part[..., h:].clone()
        part[..., :h] = a * cos - b * sin
        part[..., h:] = a * sin + b * cos
    else:
        a, b = part[..., 0::2].clone(), part[..., 1::2].clone()
        part[..., 0::2] = a * cos - b * sin
        part[..., 1::2] = a * sin + b * cos
    return y


def _rotated_rows(rows, case, positions, real):
    """Logical rows [tokens][row] with their keys turned."""
    _, hkv, dk, _, row = widths(case["model"])
    if _is_mla(case["model"]):
        return _rotated(rows[:, None], case, positions, 512, real)[:, 0]
    k = _rotated(rows[:, :hkv * dk].reshape(-1, hkv, dk), case, positions, 0, real)
    return torch.cat([k.reshape(-1, hkv * dk), rows[:, hkv * dk:].to(real)], dim=1)


# ------------------------------------------------------------------ states

class RopeState:
    def __init__(self, case, seed):
        self.case = case
        gen = torch.Generator(device="cuda").manual_seed(seed)
        T, W, at = case["tokens"], case["width"], case.get("offset", 0)
        self.positions = torch.randint(0, case["far"], (T,), generator=gen, device="cuda", dtype=torch.int32)
        if T > 64:  # a prompt: consecutive positions up to a far one
            self.positions = torch.arange(T, device="cuda", dtype=torch.int32) + max(0, case["far"] - T)
        self.src, self.dst = [], []
        for h in (int(x) for x in case["heads"].split()):
            cols = case["rot"] if at else W
            self.src.append(torch.empty(T, h, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=gen))
            self.dst.append(torch.zeros(T, h, W, dtype=torch.bfloat16, device="cuda")[..., at:])
        if own:
            from paper_2606_24506_amd import crosspool as cpl

            self.rope = cpl.Rope(device=torch.cuda.current_device(), **_rope_desc(case))
            self.parts = cpl.rope_parts(zip(self.src, self.dst))
            self.stream = torch.cuda.current_stream().cuda_stream


def _paged_segments(name, P, pages, positions):
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


class PoolState:
    """The case's requests with what they hold, and the call's buffers. The
    program holds ids, counts and device addresses ready, as a serving loop
    does."""

    def __init__(self, case, seed):
        self.case, name = case, case["model"]
        hq, hkv, dk, dv, row = widths(name)
        self.P = P = case.get("page_tokens", 64)
        self.lens = _lens(case)
        self.per = case.get("branches", 1)
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, sigma=1.0):
            return torch.empty(*shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, sigma, generator=gen)

        in_place = case["do"] == "extend"
        self.held = [normal(b + (n if in_place else 0), row, sigma=math.sqrt(0.5)) for b, n in self.lens]
        self.counts = [n for _, n in self.lens for _ in range(self.per)]
        total = sum(self.counts)
        self.rows = None if in_place else normal(total, row, sigma=math.sqrt(0.5))
        self.positions = torch.cat([torch.arange(b, b + n) for b, n in self.lens for _ in range(self.per)]).to(
            "cuda", torch.int32)
        self.q = self.out = self.lse = None
        if case["do"] != "append":
            self.q = normal(total, hq, dk)
            self.out = torch.zeros(total, hq, dv, dtype=torch.bfloat16, device="cuda")
            self.lse = torch.zeros(total, hq, device="cuda")
        self.q_in = self.q
        if case["do"] in ("step", "branch"):
            self.q_in = torch.zeros_like(self.q)
        self.slopes = self.starts = self.prefix = None
        if case.get("slopes"):
            self.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], device="cuda")
        if "docs" in case:
            spans = _spans(case)
            self.starts = torch.tensor([x for _, _, s in spans for _ in range(self.per) for x in s],
                                       dtype=torch.int32, device="cuda")
        if case.get("prefix"):
            self.prefix = [_prefix(case, b, n) for b, n in self.lens for _ in range(self.per)]
        # the pages a request holds are the lowest free ones, request by request
        held_pages = [-(-k.shape[0] // P) for k in self.held]
        new_pages = [0 if in_place else -(-(b + n) // P) - -(-b // P) for b, n in self.lens]
        branch_pages = [-(-(b + n) // P) for b, n in self.lens for _ in range(self.per)] if self.per > 1 else []
        per_chunk = CHUNK // (2 * P * row)
        pages = sum(held_pages) + (sum(branch_pages) if self.per > 1 else sum(new_pages))
        chunks = -(-pages // per_chunk) + 1
        self.mem = torch.zeros(chunks * CHUNK // 2, dtype=torch.bfloat16, device="cuda")
        self.state_out = case["do"] in ("append", "step")
        if self.state_out and not own:
            tables, k = [], 0
            for h in held_pages:
                tables.append(list(range(k, k + h)))
                k += h
            for t, m in zip(tables, new_pages):
                t += range(k, k + m)
                k += m
            segs = self.mem.view(-1, SEG)
            for t, kv in zip(tables, self.held):
                at = _paged_segments(name, P, t, torch.arange(kv.shape[0]))
                segs[at.to("cuda")] = kv.view(kv.shape[0], -1, SEG)
            self.new_at = torch.cat([_paged_segments(name, P, t, torch.arange(b, b + n))
                                     for t, (b, n) in zip(tables, self.lens)]).to("cuda")
        if own:
            self._open(name, chunks, row)
        torch.cuda.synchronize()

    def _open(self, name, chunks, row):
        from paper_2606_24506_amd import crosspool as cpl

        case = self.case
        kind, hq, hkv, d = MODELS[name]
        torch.cuda.synchronize()
        self.pool = cpl.Pool(page_tokens=self.P, pool_bytes=chunks * CHUNK, chunk_bytes=CHUNK,
                             device=torch.cuda.current_device(), device_mem=self.mem.data_ptr())
        if kind == "mla":
            m = self.pool.register(cpl.CP_KIND_MLA, hq, 1, latent_dim=512, rope_dim=64, softmax_scale=_scale(name))
        else:
            m = self.pool.register(cpl.CP_KIND_GQA, hq, hkv, head_dim=d)
        self.stream = torch.cuda.current_stream().cuda_stream
        room = 0 if self.per > 1 else 1
        held = [self.pool.open(m, max(1, kv.shape[0] + room * (0 if case["do"] == "extend" else n)))
                for kv, (_, n) in zip(self.held, self.lens)]
        for rid, kv in zip(held, self.held):
            if kv.shape[0]:
                self.pool.append([rid], [kv.shape[0]], kv, self.stream)
        self.all_ids = list(held)
        ids, drop = held, [b for b, _ in self.lens]
        if self.per > 1:
            ids = [self.pool.open(m, b + n) for b, n in self.lens for _ in range(self.per)]
            self.all_ids += ids
            self.parents = cpl.i32_array([r for r in held for _ in range(self.per)])
            drop = [0] * len(ids)
        self.ids, self.n_new = cpl.i32_array(ids), cpl.i32_array(self.counts)
        self.drop = cpl.i64_array(drop)
        self.p = [t.data_ptr() if t is not None else None for t in (self.rows, self.q_in, self.out, self.lse)]
        self.opts = dict(softcap=case.get("softcap", 0.0), window=case.get("window", 0))
        if self.slopes is not None:
            self.opts["slopes"] = self.slopes.data_ptr()
        if self.starts is not None:
            self.opts["doc_begin"] = self.starts.data_ptr()
        if self.prefix is not None:
            self.opts["prefix"] = cpl.i32_array(self.prefix)
        if case["do"] != "extend":
            self.rope = cpl.Rope(device=torch.cuda.current_device(), **_rope_desc(case))
            if self.q is not None:
                at, rot = 512 if kind == "mla" else 0, case["rot"]
                self.parts = cpl.rope_parts([(self.q, self.q_in)], offset=at)

    def __del__(self):
        pool = getattr(self, "pool", None)
        if pool is None:
            return
        torch.cuda.synchronize()
        for r in getattr(self, "all_ids", []):
            pool.close(r)
        pool.destroy()


def prepare(case, seed):
    return RopeState(case, seed) if case["do"] == "rope" else PoolState(case, seed)


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    do = s.case["do"]
    if do == "rope":
        s.rope.apply(s.parts, s.positions, stream=s.stream)
        return s.dst
    rows, q, out, lse = s.p
    if do == "append":
        s.pool.truncate(s.ids, s.drop, s.stream)
        s.pool.append_rope(s.ids, s.n_new, rows, s.rope, s.stream)
        return s.mem
    if do == "extend":
        s.pool.extend(s.ids, s.n_new, q, out, lse, s.stream, **s.opts)
        return s.out, s.lse
    s.pool.truncate(s.ids, s.drop, s.stream)
    if do == "branch":
        s.pool.fork(s.parents, s.ids, None, s.stream)
    s.rope.apply(s.parts, s.positions, stream=s.stream)
    s.pool.extend_step(s.ids, s.n_new, rows, q, out, lse, s.stream, rope=s.rope, **s.opts)
    return (s.out, s.lse, s.mem) if s.state_out else (s.out, s.lse)


# -------------------------------------------------------------- plain form

def _run_plain(s):
    case = s.case
    if case["do"] == "rope":
        return [_rotated(x, case, s.positions, 0, torch.float32).to(x.dtype) for x in s.src]
    if case["do"] == "extend":
        return _plain_attention(s, s.q, None)
    rows = _rotated_rows(s.rows, case, s.positions, torch.float32).to(torch.bfloat16)
    if s.state_out:
        s.mem.view(-1, SEG)[s.new_at] = rows.view(rows.shape[0], -1, SEG)
    if case["do"] == "append":
        return s.mem
    q = _rotated(s.q, case, s.positions, 512 if _is_mla(case["model"]) else 0, torch.float32).to(torch.bfloat16)
    got = _plain_attention(s, q, rows)
    return (*got, s.mem) if s.state_out else got


def _plain_attention(s, q, rows):
    name = s.case["model"]
    hq, hkv, dk, dv, _ = widths(name)
    g = hq // hkv
    out, lse = torch.empty_like(s.out), torch.empty_like(s.lse)
    at = 0
    for i, new in enumerate(s.counts):
        kv = s.held[i // s.per]
        if rows is not None:
            kv = torch.cat([kv, rows[at:at + new]])
        step = max(1, (1 << 28) // (g * kv.shape[0]))  # query tokens at once, for memory's sake
        for a in range(at, at + new, step):
            b = min(at + new, a + step)
            hide, far = _hidden(s, i, a, b, kv.shape[0])
            for h in range(hkv):
                k = (kv if dk != dv else kv[:, h * dk:(h + 1) * dk]).float()
                v = (kv[:, :dv] if dk != dv else kv[:, (hkv + h) * dv:(hkv + h + 1) * dv]).float()
                heads = slice(h * g, (h + 1) * g)
                x = q[a:b, heads].reshape(-1, dk).float() @ k.t().contiguous()
                x = x.view(b - a, g, -1) * _scale(name)
                if s.case.get("softcap"):
                    x = torch.tanh(x / s.case["softcap"]) * s.case["softcap"]
                if s.slopes is not None:
                    x = x - s.slopes[heads][None, :, None] * far
                x = x.masked_fill(hide, -math.inf)
                m = x.amax(dim=2, keepdim=True)
                e = torch.exp(x - m)
                z = e.sum(dim=2, keepdim=True)
                out[a:b, heads] = ((e.view((b - a) * g, -1) @ v).view(b - a, g, dv) / z).to(out.dtype)
                lse[a:b, heads] = (m + torch.log(z))[..., 0]
        at += new
    return out, lse


def _hidden(s, i, a, b, n):
    """Of query tokens [a, b), all of entry i: which of its n keys they do not
    see, and how far each is."""
    p = s.positions[a:b].long()[:, None]
    j = torch.arange(n, device="cuda")[None]
    see = j <= p
    if s.prefix is not None:
        see = see | (j < s.prefix[i])
    if s.case.get("window"):
        see = see & (j > p - s.case["window"])
    if s.starts is not None:
        see = see & (j >= s.starts[a:b].long()[:, None])
    return ~see[:, None, :], (p - j).abs().float()[:, None, :]


# ---------------------------------------------------------- 64-bit results

def _turn64(x, case, positions, offset):
    """Rotation as complex products."""
    d = _rope_desc(case)
    half = d["rot_dim"] // 2
    freq = []
    for i in range(half):
        b = d["base"]
        if d["scaling"] == "ntk":
            b = b * d["factor"] ** (d["rot_dim"] / (d["rot_dim"] - 2.0))
        f = math.pow(b, -2.0 * i / d["rot_dim"])
        if d["scaling"] == "linear":
            f /= d["factor"]
        if d["scaling"] == "parts":
            t = d["orig_len"] * f / (2 * math.pi)
            w = min(1.0, max(0.0, (t - d["low_turns"]) / (d["high_turns"] - d["low_turns"])))
            f = w * f + (1 - w) * f / d["factor"]
        freq.append(f)
    ang = torch.outer(positions.double(), torch.tensor(freq, dtype=torch.float64, device=x.device))
    turn = torch.polar(torch.full_like(ang, d["magnitude"]), ang)[:, None, :]
    y = x.double().clone()
    part = y[..., offset:offset + 2 * half]
    if d["layout"] == "half":
        z = torch.complex(part[..., :half].contiguous(), part[..., half:].contiguous()) * turn
        y[..., offset:offset + 2 * half] = torch.cat([z.real, z.imag], dim=-1)
    else:
        z = torch.view_as_complex(part.reshape(*part.shape[:-1], half, 2).contiguous()) * turn
        y[..., offset:offset + 2 * half] = torch.view_as_real(z).flatten(-2)
    return y


def _attend64(kv, q, first, lo, hi, case, slopes):
    """One request: kv [n][row], q [tokens][heads][K width], all 64-bit."""
    name = case["model"]
    hq, hkv, dk, dv, _ = widths(name)
    t, n = q.shape[0], kv.shape[0]
    lo, hi = (torch.tensor(x, device="cuda")[:, None] for x in (lo, hi))
    j = torch.arange(n, device="cuda")[None]
    outside = (j < lo) | (j >= hi)
    dist = (torch.arange(first, first + t, device="cuda")[:, None] - j).abs()
    outs, lses = [], []
    for h in range(hq):
        c = h // (hq // hkv)
        k = kv if _is_mla(name) else kv[:, c * dk:(c + 1) * dk]
        v = kv[:, :dv] if _is_mla(name) else kv[:, (hkv + c) * dv:(hkv + c + 1) * dv]
        x = torch.mm(q[:, h].contiguous(), k.t().contiguous()).mul_(_scale(name))
        if case.get("softcap"):
            x = case["softcap"] * torch.tanh(x / case["softcap"])
        if slopes is not None:
            x -= slopes[h].double() * dist
        x[outside] = -math.inf
        z = torch.logsumexp(x, dim=1, keepdim=True)
        outs.append(torch.mm(x.sub_(z).exp_(), v.contiguous()))
        lses.append(z[:, 0])
    return torch.stack(outs, 1), torch.stack(lses, 1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["do"] == "rope":
        return [_turn64(x, case, s.positions, 0) for x in s.src]
    name = case["model"]
    hq, hkv, dk, dv, row = widths(name)
    new = q = s.q
    mem = rows = None
    if case["do"] != "extend":
        if _is_mla(name):
            new = _turn64(s.rows[:, None], case, s.positions, 512)[:, 0]
        else:
            new = s.rows.double()
            new[:, :hkv * dk] = _turn64(s.rows[:, :hkv * dk].reshape(-1, hkv, dk), case, s.positions, 0).flatten(1)
        rows = new.to(torch.bfloat16)  # what the cache holds
        if s.state_out:
            mem = _mem64(case, s, new)
        if case["do"] == "append":
            return mem
        q = _turn64(s.q, case, s.positions, 512 if _is_mla(name) else 0).to(torch.bfloat16)
    outs, lses, at = [], [], 0
    for i, ((base, n), (lo, hi, _)) in enumerate(zip(s.lens, _spans(case))):
        for _ in range(s.per):
            kv = s.held[i].double()
            if rows is not None:
                kv = torch.cat([kv, rows[at:at + n].double()])
            o, e = _attend64(kv, q[at:at + n].double(), base, lo, hi, case, s.slopes)
            outs.append(o)
            lses.append(e)
            at += n
    got = (torch.cat(outs), torch.cat(lses))
    return (*got, mem) if s.state_out else got


def _mem64(case, s, new):
    """The pool's memory after the call: the held rows and, behind them, the
    new ones, each request's next page the lowest free one."""
    name, P = case["model"], s.P
    _, hkv, dk, _, row = widths(name)
    per_chunk = CHUNK // (2 * P * row)
    mem = torch.zeros(s.mem.numel(), dtype=torch.float64, device="cuda")
    free, tables, at = 0, [], 0
    for kv in s.held:
        k = (kv.shape[0] + P - 1) // P
        tables.append([free + i for i in range(k)])
        free += k
    for i, (base, n) in enumerate(s.lens):
        whole = torch.cat([s.held[i].double(), new[at:at + n]])
        at += n
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
