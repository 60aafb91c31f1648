"""Helpers of the rotary and paged-cache tests: caches whose unused rows are canaries, and the operators in float64 on
the CPU, written from their definitions.

Tolerances, by arithmetic (u = 2^-24, a rounding to fp32 is off by at most u relative):
  * rope: the angle's remainder is exact to 2^-50 turns and rounded to fp32 once (u); sine and cosine are sums whose
    terms left out are under 2^-29 and whose roundings are under 2u; a product and a fused step add 2u of |x1| + |x2|.
    Together under 8u a (|x1| + |x2|), and half a step of the output's type.
  * a logit z = scale q.k of d products added in fp32 is off by at most dz = scale (d + 2) u sum|q_i k_i|, so a
    probability by 2 dz + 16 u relative (exp2 to 1 ulp, the exponent's rounding of up to 2^6 u, the sum).  Outputs are
    off by that much of sum p|v|, plus P_ROUND of it where the probabilities are fed to the matrix units in 16 bits or
    more (fp32: all 24), plus half a step of the output's type.  Weights: by that much of each probability, and u of
    the total.
"""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2511_03092_amd as snap

U = 2.0 ** -24
P_ROUND = {"f32": 0.0, "bf16": 2.0 ** -15, "fp8": 2.0 ** -15}
KV = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}
IN = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.bfloat16}
CODE = {"f32": snap.SNAP_F32, "bf16": snap.SNAP_BF16, "fp8": snap.SNAP_FP8_E4M3}
FP8 = torch.float8_e4m3fn
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def params(hq, hkv, d, kv="bf16", latent=False, sink=4, recent=8, topk=16, **over) -> snap.Params:
    kw = dict(n_q_heads=hq, n_kv_heads=hkv, d_qk=d, d_v=512 if d == 576 else d, sink=sink, recent=recent, topk=topk,
              obs_window=1, pool_kernel=1, v_in_k=latent, in_dtype=CODE["f32" if kv == "f32" else "bf16"],
              kv_dtype=CODE[kv])
    kw.update(over)
    return snap.Params(**kw)


def canary(shape, kv):
    """Values that show when they are read: NaN in every type."""
    if kv == "fp8":
        return torch.full(shape, 0x7F, dtype=torch.uint8)
    return torch.full(shape, float("nan"), dtype=KV[kv])


class Paged:
    """One layer's paged cache on the device, with `capacity` rows of pages (in random order) for each slot that holds
    any; other pages and rows are canaries."""

    def __init__(self, p: snap.Params, kv: str, n_slots: int, page: int, capacity, seed: int, max_pages=None):
        g = torch.Generator().manual_seed(seed)
        self.p, self.kv, self.page, self.n_slots = p, kv, page, n_slots
        counts = [-(-c // page) for c in capacity]
        self.max_pages = max_pages or max(1, max(counts))
        self.n_pages = sum(counts) + 2
        order = torch.randperm(self.n_pages, generator=g).tolist()
        table = torch.full((n_slots, self.max_pages), -1, dtype=torch.int32)
        for s, m in enumerate(counts):
            for j in range(m):
                table[s, j] = order.pop()
        self.table = table.cuda()
        h = p.n_kv_heads
        self.k = canary((self.n_pages, h, page, p.d_qk), kv).cuda()
        self.v = None if p.v_in_k else canary((self.n_pages, h, page, p.d_v), kv).cuda()
        self.k_scale = self.v_scale = None
        if kv == "fp8":
            self.k_scale = (torch.rand((n_slots, h), generator=g) * 0.01 + 0.01).cuda()
            self.v_scale = None if p.v_in_k else (torch.rand((n_slots, h), generator=g) * 0.01 + 0.01).cuda()
        self.token = torch.full((self.n_pages, h, page), -7, dtype=torch.int32).cuda()
        self.weight = torch.full((self.n_pages, h, page), float("nan")).cuda()
        self.rows = torch.zeros(n_slots, dtype=torch.int32).cuda()
        self.pos = torch.zeros(n_slots, dtype=torch.int32).cuda()
        self.handle()

    def handle(self):
        self.c = snap.paged_cache_struct(self.k, self.v, self.table, self.token, self.weight, self.k_scale, self.v_scale)
        return self.c

    def state(self):
        return {x: (None if getattr(self, x) is None else getattr(self, x).cpu().clone())
                for x in ("k", "v", "token", "weight", "rows", "pos")}

    # rows [0, len) of (slot, head g) as [len, ...]; rows whose page is not there: None in `there`
    def places(self, slot, length):
        t = self.table[slot].cpu().tolist()
        return [(t[r // self.page], r % self.page) for r in range(length)]

    def gather(self, name, slot, g, length, state=None):
        x = (state[name] if state else getattr(self, name)).cpu()
        pl = self.places(slot, length)
        there = [0 <= a < self.n_pages for a, _ in pl]
        idx = torch.tensor([a if ok else 0 for (a, _), ok in zip(pl, there)], dtype=torch.long)
        off = torch.tensor([o for _, o in pl], dtype=torch.long)
        return x[idx, g, off], np.array(there, bool)

    def values(self, name, slot, g, length, state=None):
        x, there = self.gather(name, slot, g, length, state)
        if self.kv == "fp8":
            sc = (self.k_scale if name == "k" else self.v_scale)[slot, g].double().cpu()
            return x.view(FP8).double() * sc, there
        return x.double(), there


def fill(c: Paged, slots, lengths, seed, pos=None):
    """Random keys, values and weights in rows [0, length) of the slots (straight into the pages)."""
    g = torch.Generator().manual_seed(seed)
    p = c.p
    st = c.state()
    for s, n in zip(slots, lengths):
        pl = [(r, a, o) for r, (a, o) in enumerate(c.places(s, max(0, n))) if 0 <= a < c.n_pages]
        if not pl:
            continue
        r, a, o = (torch.tensor(x, dtype=torch.long) for x in zip(*pl))
        for name, d in (("k", p.d_qk), ("v", p.d_v)):
            if st[name] is None:
                continue
            x = torch.randn((len(pl), p.n_kv_heads, d), generator=g)
            st[name][a, :, o] = (x / 0.015).clamp(-448, 448).to(FP8).view(torch.uint8) if c.kv == "fp8" else x.to(KV[c.kv])
        st["weight"][a, :, o] = torch.rand((len(pl), p.n_kv_heads), generator=g)
        st["token"][a, :, o] = (r if pos is None else torch.as_tensor(pos)[r]).to(torch.int32)[:, None]
    for name in ("k", "v", "weight", "token"):
        if st[name] is not None:
            getattr(c, name).copy_(st[name])
    return c


def attend(c: Paged, slot, length, q):
    """float64 attention of q [Hq, dk] over rows [0, length): outputs [Hq, dv], probabilities [Hq, length] and the
    bounds of their errors that do not depend on the output's type."""
    p = c.p
    G, scale = p.n_q_heads // p.n_kv_heads, p.sm_scale if p.sm_scale > 0 else 1.0 / math.sqrt(p.d_qk)
    out = np.zeros((p.n_q_heads, p.d_v))
    err = np.zeros((p.n_q_heads, p.d_v))
    prob = np.zeros((p.n_q_heads, length))
    perr = np.zeros((p.n_q_heads, length))
    for g in range(p.n_kv_heads if length > 0 else 0):
        k, there = c.values("k", slot, g, length)
        v = k[:, :p.d_v] if p.v_in_k else c.values("v", slot, g, length)[0]
        k, v = k.numpy()[there], v.numpy()[there]
        if not len(k):
            continue
        for h in range(g * G, (g + 1) * G):
            qh = q[h].double().cpu().numpy()
            z = scale * (k @ qh)
            dz = scale * (p.d_qk + 2) * U * np.abs(k * qh).sum(1).max()
            e = np.exp(z - z.max())
            pr = e / e.sum()
            rel = 2 * dz + (64 + 16) * U
            prob[h, there] = pr
            perr[h, there] = rel * pr
            out[h] = pr @ v
            err[h] = (rel + P_ROUND[c.kv]) * (pr @ np.abs(v))
    return out, err, prob, perr


def rope_frequencies(r: snap.RopeParams):
    m, base = r.rot_dim, float(np.float32(r.base))
    out = []
    for i in range(m // 2):
        f = base ** (-2.0 * i / m)
        w = 1.0
        if r.rule == snap.SNAP_ROPE_DIVIDE:
            w = 0.0
        elif r.rule == snap.SNAP_ROPE_BY_TURNS:
            w = (r.orig_len * f / (2 * math.pi) - r.low_turns) / (r.high_turns - r.low_turns)
        elif r.rule == snap.SNAP_ROPE_BY_INDEX:
            at = lambda t: m * math.log(r.orig_len / (2 * math.pi * t)) / (2 * math.log(base))  # noqa: E731
            lo, hi = max(0, math.floor(at(r.high_turns))), min(m - 1, math.ceil(at(r.low_turns)))
            w = 1.0 - (i - lo) / max(hi - lo, 0.001)
        w = min(1.0, max(0.0, w))
        out.append(w * f + (1.0 - w) * f / (r.factor if r.rule else 1.0))
    return np.array(out)


def rope(r: snap.RopeParams, x, position):
    """x [..., d] (float64) at positions [...]: the turned heads and |x1| + |x2| of every rotated dim."""
    ang = position[..., None] * rope_frequencies(r)
    c, s = r.amplitude * np.cos(ang), r.amplitude * np.sin(ang)
    i = np.arange(r.rot_dim // 2)
    one = r.rot_start + (2 * i if r.layout == snap.SNAP_ROPE_PAIRS else i)
    two = one + (1 if r.layout == snap.SNAP_ROPE_PAIRS else r.rot_dim // 2)
    y, size = x.copy(), np.zeros_like(x)
    y[..., one] = x[..., one] * c - x[..., two] * s
    y[..., two] = x[..., two] * c + x[..., one] * s
    size[..., one] = size[..., two] = np.abs(x[..., one]) + np.abs(x[..., two])
    return y, r.amplitude * size


def evict(token, weight, rows, pos, sink, recent, budget):
    """The row whose contents end in each row [0, budget) (-1 past the rows held), for one (slot, head)."""
    if rows <= budget:
        return np.array([r if r < rows else -1 for r in range(budget)], dtype=np.int64)
    w = np.where(np.isnan(weight) | (weight < 0), 0.0, weight)
    safe = (token < sink) | (token >= pos - recent)
    kept = np.flatnonzero(safe)[:budget].tolist()
    others = sorted(np.flatnonzero(~safe).tolist(), key=lambda r: (-w[r], r))
    kept = sorted(kept + others[:max(0, budget - int(safe.sum()))])
    out = np.full(budget, -1, dtype=np.int64)
    here = [r for r in kept if r < budget]
    out[here] = here
    out[np.flatnonzero(out < 0)] = [r for r in kept if r >= budget]
    return out
