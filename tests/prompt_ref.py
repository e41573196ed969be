"""Plain 64-bit forms of rotary positions and of attention of token chunks,
and a pool with the rows its requests hold, for the tests of those operators."""
from __future__ import annotations

import math

import numpy as np
import torch

from paper_2606_24506_amd import crosspool as cpl

GEOMS = {
    "gqa8x2d128": dict(kind=cpl.CP_KIND_GQA, n_q_heads=8, n_kv_heads=2, head_dim=128),
    "gqa6x2d64": dict(kind=cpl.CP_KIND_GQA, n_q_heads=6, n_kv_heads=2, head_dim=64),
    "mha3d64": dict(kind=cpl.CP_KIND_GQA, n_q_heads=3, n_kv_heads=3, head_dim=64),
    "mqa32d128": dict(kind=cpl.CP_KIND_GQA, n_q_heads=32, n_kv_heads=1, head_dim=128),
    "gqa5x1d128": dict(kind=cpl.CP_KIND_GQA, n_q_heads=5, n_kv_heads=1, head_dim=128),
    "gqa4x2d256": dict(kind=cpl.CP_KIND_GQA, n_q_heads=4, n_kv_heads=2, head_dim=256),
    "mha2d512": dict(kind=cpl.CP_KIND_GQA, n_q_heads=2, n_kv_heads=2, head_dim=512),
    "mla16": dict(kind=cpl.CP_KIND_MLA, n_q_heads=16, n_kv_heads=1, latent_dim=512, rope_dim=64, softmax_scale=0.0722),
    "mla20": dict(kind=cpl.CP_KIND_MLA, n_q_heads=20, n_kv_heads=1, latent_dim=512, rope_dim=64, softmax_scale=0.0722),
    "mla128": dict(kind=cpl.CP_KIND_MLA, n_q_heads=128, n_kv_heads=1, latent_dim=512, rope_dim=64,
                   softmax_scale=0.0722),
    "mla4l128r40": dict(kind=cpl.CP_KIND_MLA, n_q_heads=4, n_kv_heads=1, latent_dim=128, rope_dim=40,
                        softmax_scale=0.1),
    "mla4l64r0": dict(kind=cpl.CP_KIND_MLA, n_q_heads=4, n_kv_heads=1, latent_dim=64, rope_dim=0, softmax_scale=0.1),
}


def shape(name):
    """(query heads, KV heads, K width, V width, row elements, scale)"""
    g = GEOMS[name]
    if g["kind"] == cpl.CP_KIND_MLA:
        dk = g["latent_dim"] + g["rope_dim"]
        return g["n_q_heads"], 1, dk, g["latent_dim"], dk, g["softmax_scale"]
    d = g["head_dim"]
    return g["n_q_heads"], g["n_kv_heads"], d, d, 2 * d * g["n_kv_heads"], 1 / math.sqrt(d)


def turn(x, angles, positions, layout, magnitude=1.0, inverse=False):
    """x [tokens][heads][rot] in 64 bits, turned by positions x angles."""
    x = x.double().cpu()
    ang = positions.double().cpu()[:, None, None] * torch.as_tensor(angles, dtype=torch.float64)
    if inverse:
        ang = -ang
    c, s = torch.cos(ang) * magnitude, torch.sin(ang) * magnitude
    h = x.shape[-1] // 2
    y = torch.empty_like(x)
    a, b = (x[..., :h], x[..., h:]) if layout == "half" else (x[..., 0::2], x[..., 1::2])
    u, w = a * c - b * s, a * s + b * c
    if layout == "half":
        y[..., :h], y[..., h:] = u, w
    else:
        y[..., 0::2], y[..., 1::2] = u, w
    return y


def turn_rows(name, rows, angles, positions, layout):
    """Logical rows [tokens][row] with their keys turned, in 64 bits."""
    _, hkv, dk, dv, _, _ = shape(name)
    rot = 2 * len(angles)
    y = rows.double().cpu().clone()
    if GEOMS[name]["kind"] == cpl.CP_KIND_MLA:
        y[:, dv:dv + rot] = turn(y[:, None, dv:dv + rot], angles, positions, layout)[:, 0]
    else:
        k = y[:, :hkv * dk].view(-1, hkv, dk)
        k[..., :rot] = turn(k[..., :rot], angles, positions, layout)
    return y


def attend(name, rows, q, softcap=0.0, window=0, slopes=None, prefix=0, doc_begin=None):
    """rows [context][row], q [tokens][heads][K width] -> out, lse in 64 bits,
    and sum p |v| of each output. Rows that see nothing: 0 and -inf."""
    hq, hkv, dk, dv, _, scale = shape(name)
    rows, q = rows.double().cpu(), q.double().cpu()
    n, t = rows.shape[0], q.shape[0]
    pos = torch.arange(n - t, n)[:, None]
    j = torch.arange(n)[None]
    see = j < torch.maximum(pos + 1, torch.tensor(min(prefix, n)))
    if window:
        see &= j > pos - window
    if doc_begin is not None:
        see &= j >= doc_begin.cpu().long()[:, None]
    out, lse, mag = (torch.zeros(t, hq, dv, dtype=torch.float64), torch.zeros(t, hq, dtype=torch.float64),
                     torch.zeros(t, hq, dv, dtype=torch.float64))
    mla = GEOMS[name]["kind"] == cpl.CP_KIND_MLA
    for h in range(hq):
        c = h // (hq // hkv)
        k = rows if mla else rows[:, c * dk:(c + 1) * dk]
        v = rows[:, :dv] if mla else rows[:, (hkv + c) * dv:(hkv + c + 1) * dv]
        for i in range(t):  # only what the row sees enters
            idx = see[i].nonzero()[:, 0]
            if len(idx) == 0:
                lse[i, h] = -math.inf
                continue
            s = (k[idx] @ q[i, h]) * scale
            if softcap:
                s = softcap * torch.tanh(s / softcap)
            if slopes is not None:
                s = s - float(slopes[h]) * (pos[i] - idx).abs().double()
            lse[i, h] = torch.logsumexp(s, 0)
            p = torch.exp(s - lse[i, h])
            out[i, h] = p @ v[idx]
            mag[i, h] = p @ v[idx].abs()
    return out, lse, mag


HALF_BF16 = 2.0 ** -8  # a rounding to bf16 is off by at most this part of the value


def check(got_out, got_lse, ref, p_bits16, label=""):
    """Outputs against the 64-bit form. Allowed: the output's rounding, 2^-8
    of it; the probabilities' rounding, 2^-8 (prompt chunks on the matrix
    cores) or 2^-16 (two bf16 parts, or fp32) of sum p |v|; and for what 32 bits
    lose 2^-12 of sum p |v| (scores of up to 2^6 held to 2^-24 of themselves and a
    product's 576 additions each 2^-24 of at most 2^6: below 2^-9 in the worst
    case, where every error has one sign, and 2^-13 for the roots of their
    count), the same for lse, plus 2^-22 of it."""
    out, lse, mag = ref
    got_out, got_lse = got_out.double().cpu(), got_lse.double().cpu()
    tol = HALF_BF16 * out.abs() + ((2.0 ** -8 if p_bits16 else 0.0) + 2.0 ** -12) * mag + 1e-30
    err = (got_out - out).abs()
    worst = (err / tol).max().item()
    empty = torch.isinf(lse)
    assert torch.equal(torch.isinf(got_lse) & (got_lse < 0), empty), label
    lerr = torch.where(empty, 0.0, (got_lse - lse).abs())
    lworst = (lerr / (2.0 ** -12 + 2.0 ** -22 * torch.where(empty, 0.0, lse.abs()))).max().item()
    print(f"[extend] {label} out {worst:.3f} lse {lworst:.3f} of the tolerance", flush=True)
    assert torch.isfinite(got_out).all(), label
    assert worst <= 1 and lworst <= 1, (label, worst, lworst)


class Scene:
    """A pool with one model and requests holding random rows."""

    def __init__(self, name, lens, page_tokens=64, seed=0, room=0, device=0, fill=None, layers=1, **pool):
        self.name = name
        self.hq, self.hkv, self.dk, self.dv, self.row, _ = shape(name)
        gen = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.gen = gen
        need = sum(-(-(n + room) // page_tokens) for n in lens) * 2 * page_tokens * self.row * layers
        chunk = pool.pop("chunk_bytes", 2 << 20)
        self.pool_bytes = pool.pop("pool_bytes", need * 2 + (8 + len(lens)) * chunk)
        if fill is not None:  # stale memory
            self.mem = torch.full((self.pool_bytes // 2,), fill, dtype=torch.bfloat16, device="cuda")
            torch.cuda.synchronize()
            pool["device_mem"] = self.mem.data_ptr()
        self.pool = cpl.Pool(page_tokens=page_tokens, pool_bytes=self.pool_bytes, chunk_bytes=chunk,
                             placement_seed=seed + 3, device=device, **pool)
        self.model = self.pool.register(**GEOMS[name], n_layers=layers)
        self.ids, self.rows = [], []
        for n in lens:
            self.add(n, room, layers)

    def normal(self, *shape, sigma=1.0):
        return torch.empty(*shape, dtype=torch.bfloat16, device="cuda").normal_(0, sigma, generator=self.gen)

    def add(self, n, room=0, layers=1):
        rows = self.normal(layers, n, self.row, sigma=0.7)
        rid = self.pool.open(self.model, max(1, n + room))
        if n:
            self.pool.append([rid], [n], rows)
        self.ids.append(rid)
        self.rows.append(rows[0] if layers == 1 else rows)
        return rid

    def buffers(self, total):
        return (self.normal(total, self.hq, self.dk), torch.full((total, self.hq, self.dv), 7.0, dtype=torch.bfloat16,
                                                                device="cuda"),
                torch.full((total, self.hq), 7.0, device="cuda"))

    def held(self, rid, n, layers=1):
        """The request's logical rows, out of the pool."""
        dst = torch.zeros(layers, n, self.row, dtype=torch.bfloat16, device="cuda")
        if n:
            self.pool.gather(rid, 0, n, dst)
        return dst if layers > 1 else dst[0]

    def close(self):
        torch.cuda.synchronize()
        for r in self.ids:
            self.pool.close(r)
        self.pool.destroy()


def rounds_to_16_bits(name, n_q, path=cpl.CP_PATH_AUTO):
    """Does this request's kernel round probabilities to bf16?"""
    g = GEOMS[name]
    if path == cpl.CP_PATH_VALU:
        return False
    if g["kind"] == cpl.CP_KIND_GQA and g["head_dim"] in (64, 128):
        return n_q * g["n_q_heads"] // g["n_kv_heads"] > 32
    return g["kind"] == cpl.CP_KIND_MLA and (g["latent_dim"], g["rope_dim"]) == (512, 64)


def bits(x):
    return x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
