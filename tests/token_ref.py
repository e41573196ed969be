"""Plain 64-bit forms of attention over drafted trees, of the weight that queries
give to cached tokens and of the choice of tokens to keep, for the tests of those
operators."""
from __future__ import annotations

import math
import random

import torch

from paper_2606_24506_amd import crosspool as cpl
from prompt_ref import GEOMS, shape


def make_tree(n, seed, width=6, roots=0.1):
    """Parents of a random tree of n tokens."""
    rng = random.Random(seed)
    return [-1 if t == 0 or rng.random() < roots else rng.randrange(max(0, t - width), t) for t in range(n)]


def ancestors(parents):
    """(sees [n][n], depth [n]) by walking up."""
    n = len(parents)
    sees, depth = torch.zeros(n, n, dtype=torch.bool), torch.zeros(n, dtype=torch.int32)
    for t in range(n):
        a, d = t, -1
        while a >= 0:
            sees[t, a] = True
            d += 1
            a = parents[a] if 0 <= parents[a] < a else -1
        depth[t] = d
    return sees, depth


def pack(sees, words):
    """[n][words] int32 masks of a bool [n][m]."""
    n, m = sees.shape
    out = torch.zeros(n, words * 32, dtype=torch.int64)
    out[:, :m] = sees.long()
    w = (out.view(n, words, 32) << torch.arange(32)).sum(2)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def heads_of(name, rows, h):
    """K and V rows of query head h, in 64 bits."""
    hq, hkv, dk, dv, _, _ = shape(name)
    rows = rows.double().cpu()
    if GEOMS[name]["kind"] == cpl.CP_KIND_MLA:
        return rows, rows[:, :dv]
    c = h // (hq // hkv)
    return rows[:, c * dk:(c + 1) * dk], rows[:, (hkv + c) * dv:(hkv + c + 1) * dv]


def attend_tree(name, rows, q, sees, depth, softcap=0.0, window=0, slopes=None, doc_begin=None):
    """As prompt_ref.attend, of a tree whose tokens are the last of the rows."""
    hq, _, _, dv, _, scale = shape(name)
    n, t = rows.shape[0], q.shape[0]
    base = n - t
    q = q.double().cpu()
    stand = torch.cat([torch.arange(base), base + depth.long().cpu()])
    out, lse, mag = (torch.zeros(t, hq, dv, dtype=torch.float64), torch.zeros(t, hq, dtype=torch.float64),
                     torch.zeros(t, hq, dv, dtype=torch.float64))
    for i in range(t):
        p = int(stand[base + i])
        lo = max(0, p - window + 1) if window else 0
        if doc_begin is not None:
            lo = max(lo, int(doc_begin[i]))
        see = torch.zeros(n, dtype=torch.bool)
        see[min(lo, base):base] = True
        see[base:] = sees[i, :t]
        idx = see.nonzero()[:, 0]
        for h in range(hq):
            if len(idx) == 0:
                lse[i, h] = -math.inf
                continue
            k, v = heads_of(name, rows, h)
            s = (k[idx] @ q[i, h]) * scale
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            if slopes is not None:
                s = s - float(slopes[h]) * (p - stand[idx]).abs().double()
            lse[i, h] = torch.logsumexp(s, 0)
            w = torch.exp(s - lse[i, h])
            out[i, h] = w @ v[idx]
            mag[i, h] = w @ v[idx].abs()
    return out, lse, mag


def given(name, rows, q, lse, softcap=0.0, window=0, slopes=None, prefix=0, doc_begin=None):
    """The weight that the queries of the rows' last tokens give to each row, per KV
    head, in 64 bits: e^(s - lse) of what they see."""
    hq, hkv, _, _, _, scale = shape(name)
    n, t = rows.shape[0], q.shape[0]
    q, lse = q.double().cpu(), lse.double().cpu()
    pos = torch.arange(n - t, n)[:, None]
    j = torch.arange(n)[None]
    see = j < torch.maximum(pos + 1, torch.tensor(min(prefix, n)))
    if window:
        see &= j > pos - window
    if doc_begin is not None:
        see &= j >= doc_begin.cpu().long()[:, None]
    out = torch.zeros(hkv, n, dtype=torch.float64)
    for h in range(hq):
        k, _ = heads_of(name, rows, h)
        s = (q[:, h] @ k.t()) * scale
        if softcap:
            s = softcap * torch.tanh(s / softcap)
        if slopes is not None:
            s = s - float(slopes[h]) * (pos - j).abs().double()
        w = torch.where(see & (lse[:, h] != -math.inf)[:, None], torch.exp(s - lse[:, h, None]), 0.0)
        out[h // (hq // hkv)] += w.sum(0)
    return out


def heaviest(w, keep, first, last):
    """Numbers of the tokens of one row of weights that stay, rising."""
    n = len(w)
    if keep >= n:
        return list(range(n))
    middle = [(x != x, -x if x == x else 0.0, t) for t, x in enumerate(w)][first:n - last]  # NaN behind -inf
    chosen = sorted(middle)[:keep - first - last]
    return list(range(first)) + sorted(c[2] for c in chosen) + list(range(n - last, n))


def kept_rows(name, rows, kept):
    """rows [layers][n][row] cut to kept [layers][KV heads][keep]."""
    _, hkv, dk, dv, row, _ = shape(name)
    out = torch.zeros(rows.shape[0], len(kept[0][0]), row, dtype=rows.dtype)
    rows = rows.cpu()
    for l in range(rows.shape[0]):
        for h in range(hkv):
            idx = torch.tensor(kept[l][h], dtype=torch.int64)
            if GEOMS[name]["kind"] == cpl.CP_KIND_MLA:
                out[l] = rows[l][idx]
            else:
                for part in (h, hkv + h):
                    out[l][:, part * dk:(part + 1) * dk] = rows[l][idx][:, part * dk:(part + 1) * dk]
    return out
