"""Helpers of the block-cache tests: a cache whose unused parts are canaries, the rows that were put into it, and the
operators from their definitions on the CPU (codes and scores in the 32-bit steps that define them, attention in float64).

Tolerances, by arithmetic (u = 2^-24): codes, scales, bounds, tails and selections are exact.  A logit z = scale s q.c of d
products (codes c, scale s) added in fp32 is off by at most dz = scale s (d + 2) u sum|q_i c_i| and two roundings of its
factors, so a probability by 2 dz + 16 u relative (exp2 to 1 ulp, the exponent's rounding of up to 2^6 u, the sum), outputs
by that much of sum p|v|, plus 2^-18 of it where probabilities enter the value product in 16-bit terms, plus half a step of
the output's type."""
from __future__ import annotations

import math

import numpy as np
import torch

import paper_2511_03092_amd as snap
from pagedhelp import FP8, HALF_STEP, U

KIND = {"bf16": (snap.SNAP_BF16, torch.bfloat16), "fp8": (snap.SNAP_FP8_E4M3, torch.uint8), "i8": (snap.SNAP_INT8, torch.int8)}
TOP = {"fp8": 448.0, "i8": 127.0}


def params(hq, hkv, d, kv="i8", **over) -> snap.Params:
    kw = dict(n_q_heads=hq, n_kv_heads=hkv, d_qk=d, d_v=d, sink=4, recent=8, topk=16, obs_window=1, pool_kernel=1,
              in_dtype=snap.SNAP_BF16, kv_dtype=KIND[kv][0])
    kw.update(over)
    return snap.Params(**kw)


def amax(x):
    """Largest finite magnitude of the last two dims, float32."""
    x = x.float().abs()
    return torch.where(torch.isfinite(x), x, torch.zeros_like(x)).amax((-2, -1))


def scale_of(x, top):
    m = amax(x)
    s = (m * (1.0 / torch.tensor(top, dtype=torch.float32))).clamp(min=2.0 ** -126)
    return torch.where(m == 0, torch.ones_like(s), s)


def codes_of(x, kv):
    """x [..., block, d] bf16 -> codes (bytes as stored), scales."""
    s = scale_of(x, TOP[kv])
    y = x.float() / s[..., None, None]
    nan = torch.isnan(y)
    y = torch.where(nan, torch.zeros_like(y), y.clamp(-TOP[kv], TOP[kv]))
    if kv == "i8":
        return torch.round(y).to(torch.int8), s
    c = y.to(FP8).view(torch.uint8)
    return torch.where(nan, torch.full_like(c, 0x7F), c), s


def bounds_of(x):
    s = scale_of(x, 127.0)
    f = x.float()
    nan = torch.isnan(f)
    none = nan.all(-2)
    lo = torch.where(nan, torch.full_like(f, math.inf), f).amin(-2)
    hi = torch.where(nan, torch.full_like(f, -math.inf), f).amax(-2)
    both = torch.stack(((lo / s[..., None]).floor(), (hi / s[..., None]).ceil()), -2).clamp(-127, 127)
    return torch.where(none[..., None, :], torch.zeros_like(both), both).to(torch.int8), s


class Blocks:
    """One layer's block cache on the device with `capacity` rows of pages for each slot, and what was put into it."""

    def __init__(self, p, kv, block, page, capacity, seed, bounds=True, holes=(), n_pages=None, max_pages=None):
        g = torch.Generator().manual_seed(seed)
        self.p, self.kv, self.block, self.page, self.n_slots = p, kv, block, page, len(capacity)
        counts = [-(-c // page) for c in capacity]
        self.max_pages = max_pages or max(1, max(counts))
        used = sum(counts)
        self.n_pages = n_pages or used + 2
        order = (self.n_pages - 1 - torch.randperm(used + 2, generator=g)).tolist()
        self.table_cpu = torch.full((self.n_slots, self.max_pages), -1, dtype=torch.int32)
        for s, m in enumerate(counts):
            for j in range(m):
                self.table_cpu[s, j] = order.pop()
        for i, (s, j) in enumerate(holes):
            self.table_cpu[s, j] = (-1, self.n_pages, 2 ** 31 - 1, -2 ** 31)[i % 4]
        self.table = self.table_cpu.cuda()
        h, d, per = p.n_kv_heads, p.d_qk, page // block
        dt = KIND[kv][1]
        fill = {"bf16": float("nan"), "fp8": 0x7F, "i8": 85}[kv]
        self.k, self.v = (torch.full((self.n_pages, h, page, d), fill, dtype=dt, device="cuda") for _ in range(2))
        eight = kv != "bf16"
        nan = float("nan")
        self.k_scale, self.v_scale = (torch.full((self.n_pages, h, per), nan, device="cuda") if eight else None for _ in range(2))
        self.k_tail, self.v_tail = (torch.full((self.n_slots, h, block, d), nan, dtype=torch.bfloat16, device="cuda") if eight
                                    else None for _ in range(2))
        self.bound = torch.full((self.n_pages, h, per, 2, d), 99, dtype=torch.int8, device="cuda") if bounds else None
        self.bound_scale = torch.full((self.n_pages, h, per), nan, device="cuda") if bounds else None
        self.rows = torch.zeros(self.n_slots, dtype=torch.int32, device="cuda")
        self.x = {n: [torch.zeros((0, h, d), dtype=torch.bfloat16) for _ in range(self.n_slots)] for n in ("k", "v")}
        self.c = snap.block_cache_struct(self.k, self.v, self.table, block, self.k_scale, self.v_scale, self.k_tail,
                                         self.v_tail, self.bound, self.bound_scale)

    NAMES = ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "bound", "bound_scale")

    def state(self):
        return {n: getattr(self, n).cpu().clone() for n in self.NAMES if getattr(self, n) is not None}

    def put(self, slot, k, v):
        """Notes rows [len, h, d] as stored behind the slot's (not on the device)."""
        room = self.max_pages * self.page - len(self.x["k"][slot])
        for n, y in (("k", k), ("v", v)):
            self.x[n][slot] = torch.cat((self.x[n][slot], y[:max(0, room)].cpu()))

    def there(self, slot, block):
        j = block * self.block // self.page
        if j >= self.max_pages:
            return -1
        page = int(self.table_cpu[slot, j])
        return page if 0 <= page < self.n_pages else -1

    def check(self, before):
        """Everything on the device against the rows put in; what was not written is as in `before`."""
        want = {n: t.clone() for n, t in before.items()}
        got = self.state()
        B, per = self.block, self.page // self.block
        for slot in range(self.n_slots):
            for n in ("k", "v"):
                x = self.x[n][slot]
                for j in range(-(-len(x) // B)):
                    page = self.there(slot, j)
                    if page < 0:
                        continue
                    y = x[j * B:(j + 1) * B].transpose(0, 1)  # [h, rows, d]
                    a = j % per
                    if self.kv == "bf16":
                        want[n][page, :, a * B:a * B + y.shape[1]] = y
                    elif y.shape[1] == B:
                        codes, s = codes_of(y, self.kv)
                        want[n][page, :, a * B:(a + 1) * B] = codes
                        want[n + "_scale"][page, :, a] = s
                    if n == "k" and self.bound is not None and y.shape[1] == B:
                        want["bound"][page, :, a], want["bound_scale"][page, :, a] = bounds_of(y)
                if self.kv != "bf16" and len(x) and self.there(slot, (len(x) - 1) // B) >= 0:
                    m = (len(x) - 1) % B
                    last = x[len(x) - 1 - m:].transpose(0, 1)
                    assert torch.equal(got[n + "_tail"][slot, :, :m + 1].view(torch.int16), last.contiguous().view(torch.int16)), (n, slot)
        for n in want:
            if n.endswith("_tail"):
                continue
            a, b = got[n].contiguous().view(torch.uint8), want[n].contiguous().view(torch.uint8)
            assert torch.equal(a, b), (n, int((a != b).sum()))
        return got

    def values(self, n, slot, g, blocks):
        """Rows of whole blocks as the cache holds them, float64 [rows, d]."""
        x = torch.cat([self.x[n][slot][j * self.block:(j + 1) * self.block, g] for j in blocks]) if len(blocks) else \
            torch.zeros((0, self.p.d_qk), dtype=torch.bfloat16)
        if self.kv == "bf16" or not len(blocks):
            return x.double()
        x = x.view(len(blocks), self.block, -1)
        codes, s = codes_of(x, self.kv)
        v = codes.view(FP8).double() if self.kv == "fp8" else codes.double()
        return (v * s.double()[:, None, None]).flatten(0, 1)


def scores(c: Blocks, slot, g, q, blocks):
    """float32 scores of blocks for the group's queries q [G, d], in the steps that define them."""
    f = q.float()
    u = scale_of(f[:, None], 127.0)
    y = f / u[:, None]
    a = torch.where(torch.isnan(y), torch.zeros_like(y), torch.round(y.clamp(-127, 127))).double()
    out = []
    for j in blocks:
        b, s = bounds_of(c.x["k"][slot][j * c.block:(j + 1) * c.block, g])
        dots = torch.where(a > 0, a * b[1].double(), a * b[0].double()).sum(1)
        out.append(float(((dots.float() * u).max() * s)))
    return np.array(out, dtype=np.float32)


def choose(c: Blocks, slot, g, r, q, max_rows):
    """Selected blocks for the newest row r."""
    p, B = c.p, c.block
    n = (r if r < max_rows else max_rows) // B
    forced = [j for j in range(n) if (j * B < p.sink or (j + 1) * B > r + 1 - p.recent)]
    other = [j for j in range(n) if j not in set(forced) and c.there(slot, j) >= 0]
    forced = [j for j in forced if c.there(slot, j) >= 0]
    k = -(-p.topk // B)
    if len(other) > k:
        s = scores(c, slot, g, q, other)
        order = sorted(range(len(other)), key=lambda i: (-float(s[i]), i))[:k]
        other = [other[i] for i in order]
    return sorted(forced + other)


def attend(c: Blocks, slot, r, q, max_rows, select):
    """Outputs [Hq, d] in float64, the bounds of their errors (but the output's rounding), and the selections."""
    p, B = c.p, c.block
    G, d = p.n_q_heads // p.n_kv_heads, p.d_qk
    scale = p.sm_scale if p.sm_scale > 0 else 1.0 / math.sqrt(d)
    out, err, sel = np.zeros((p.n_q_heads, d)), np.zeros((p.n_q_heads, d)), []
    for g in range(p.n_kv_heads):
        if r < 0:
            sel.append([])
            continue
        n = (r if r < max_rows else max_rows) // B
        blocks = choose(c, slot, g, r, q[g * G:(g + 1) * G].cpu(), max_rows) if select else \
            [j for j in range(n) if c.there(slot, j) >= 0]
        sel.append(blocks)
        T = r // B
        tail = r < max_rows and c.there(slot, T) >= 0
        k, v = (torch.cat((c.values(x, slot, g, blocks), c.x[x][slot][T * B:r + 1, g].double() if tail else
                           torch.zeros((0, d), dtype=torch.float64))).numpy() for x in ("k", "v"))
        if not len(k):
            continue
        for h in range(g * G, (g + 1) * G):
            qh = q[h].double().cpu().numpy()
            z = scale * (k @ qh)
            dz = scale * (d + 4) * U * np.abs(k * qh).sum(1).max()
            e = np.exp(z - z.max())
            pr = e / e.sum()
            out[h] = pr @ v
            err[h] = (2 * dz + (64 + 16) * U + 2.0 ** -18) * (pr @ np.abs(v))
    return out, err, sel


def check_out(c: Blocks, slots, rows, q, out, max_rows, select=False, sel_out=None, only=None):
    """A call's outputs (and selections) against the definition; rows: each slot's newest row (None: no such slot)."""
    for b, (s, r) in enumerate(zip(slots, rows)):
        if only is not None and b not in only:
            continue
        want, err, sel = attend(c, s, -1 if r is None else r, q[b], max_rows, select)
        got = out[b].double().cpu().numpy()
        tol = err + HALF_STEP[out.dtype] * (np.abs(want) + err) + 1e-30
        bad = np.abs(got - want) > tol
        assert not bad.any(), (b, s, r, np.abs(got - want)[bad].max(), (np.abs(got - want) / tol).max())
        if select and sel_out is not None:
            for g, w in enumerate(sel):
                have = sel_out[b, g].cpu().tolist()
                assert have == w + [-1] * (len(have) - len(w)), (b, g, have, w)
