"""Rotary positions and the paged cache (store, attention of one new token, eviction), as a serving program calls them:
sizes, what is in hand before a call, the call, and what it has to give.

Four kinds of case:

  rope    rotary positions applied to the queries and keys of a step or of a prompt.  Prompts come as a projection
          leaves them, token by token with the heads of q, k and v side by side, and go to the head-by-head layout that
          prefill attention takes; the rotated part of latent rows goes into its place at their end.
  append  new tokens' keys and values stored into a paged cache: one token for each sequence, or whole prompts with the
          weights that prompt scoring gave their tokens.
  decode  a new token is stored, and its queries attend every row of their sequence; with ``weigh`` each row's softmax
          weights, summed over the query heads that share it, are added to the row's accumulated weight.
  evict   a sequence that has outgrown its budget keeps its first and latest tokens and the heaviest others.

``plain_*`` are the same operators in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
IN_T = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.bfloat16}
KV_T = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}
FP8 = torch.float8_e4m3fn
ELT = {"f32": 4, "bf16": 2, "fp8": 1}


# ---------------------------------------------------------------- cases
def _rope(*, n, tokens, hq, hkv, d, into=None, start=0, rot=None, pairs=False, rule="plain", base=500000.0, factor=1.0,
          far=0, kv="bf16", packed=False, ragged=False, **name):
    return dict(op="rope", n=n, tokens=tokens, hq=hq, hkv=hkv, d=d, into=d if into is None else into, start=start,
                rot=d if rot is None else rot, pairs=pairs, rule=rule, base=base, factor=factor, far=far, kv=kv,
                packed=packed, ragged=ragged, **name)


def _append(*, n, tokens, hkv, d, dv=None, latent=False, kv="bf16", page=64, held=0, weighted=False, packed=False,
            ragged=False, **name):
    return dict(op="append", n=n, tokens=tokens, hkv=hkv, d=d, dv=d if dv is None else dv, latent=latent, kv=kv,
                page=page, held=held, weighted=weighted, packed=packed, ragged=ragged, **name)


def _decode(*, n, rows, hq, hkv, d, dv=None, latent=False, kv="bf16", page=64, weigh=False, ragged=False, **name):
    return dict(op="decode", n=n, rows=rows, hq=hq, hkv=hkv, d=d, dv=d if dv is None else dv, latent=latent, kv=kv,
                page=page, weigh=weigh, ragged=ragged, **name)


def _evict(*, n, rows, hkv, d, dv=None, latent=False, kv="bf16", page=64, sink=4, recent, topk, mixed=False, **name):
    return dict(op="evict", n=n, rows=rows, hkv=hkv, d=d, dv=d if dv is None else dv, latent=latent, kv=kv, page=page,
                sink=sink, recent=recent, topk=topk, mixed=mixed, **name)


def listed():
    return [
        # One decode step of 16 sequences far into a long context (frequencies stretched for it): the smallest call, one
        # per layer and token.
        _rope(name="rope-step-16", n=16, tokens=1, hq=32, hkv=8, d=128, rule="turns", factor=8.0, far=120000),
        # A 32k Llama-shaped prompt out of the packed projection, into the layout of prefill attention.
        _rope(name="rope-prompt-32k", n=1, tokens=32768, hq=32, hkv=8, d=128, packed=True),
        # Latent rows: the last 64 of 576 dims, interleaved pairs, ragged prompts of odd lengths.
        _rope(name="rope-latent-3x9k", n=3, tokens=9001, hq=8, hkv=1, d=64, into=576, pairs=True, rule="index",
              base=10000.0, factor=40.0, packed=True, ragged=True),
        # One token for each of 32 fp8 sequences: a continuous-batching step of one layer.
        _append(name="append-step-fp8-32", n=32, tokens=1, hkv=8, d=128, kv="fp8", held=8191),
        # Four ragged prompts of up to 32k tokens with their prompt weights, out of the packed projection.
        _append(name="append-prompt-4x32k", n=4, tokens=32768, hkv=8, d=128, packed=True, weighted=True, ragged=True),
        # One short conversation: latency and launches are all there is to it.
        _decode(name="decode-1x500", n=1, rows=500, hq=32, hkv=8, d=128, page=16),
        # Eight uncompressed contexts from a few thousand to 128k tokens, with the weights that eviction goes by.
        _decode(name="decode-8x128k-weigh", n=8, rows=131072, hq=32, hkv=8, d=128, weigh=True, ragged=True),
        # Continuous batching over fp8 pages: 32 sequences of unequal length.
        _decode(name="decode-fp8-32x16k-weigh", n=32, rows=16384, hq=32, hkv=8, d=128, kv="fp8", weigh=True,
                ragged=True),
        # One GPU's head share of a latent-cache (MLA) model, 16 sequences of 32k.
        _decode(name="decode-latent-16x32k", n=16, rows=32768, hq=8, hkv=1, d=576, dv=512, latent=True),
        # A small fp32 model, rows that end inside a page.
        _decode(name="decode-f32-3x1001", n=3, rows=1001, hq=4, hkv=2, d=64, kv="f32", page=32, weigh=True),
        # A 32k prompt cut to a 4096-row budget.
        _evict(name="evict-1x32k-to-4k", n=1, rows=32768, hkv=8, d=128, recent=1024, topk=3068),
        # Eight sequences back to their 16384-row budget after 1500 more tokens, rows in the order earlier evictions
        # left them.
        _evict(name="evict-8x18k-to-16k", n=8, rows=17884, hkv=8, d=128, recent=2048, topk=14332, mixed=True),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, its logarithm spread evenly."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """One more case: batch, length, heads, width, type, page size and layout drawn apart, at most the work of the
    largest listed case."""
    op = rng.choice(("rope", "append", "decode", "decode", "evict"))
    heads, d = rng.choice((((32, 8), 128), ((8, 8), 64), ((16, 1), 128), ((24, 8), 128), ((4, 2), 64), ((16, 2), 64),
                           ((8, 1), 576), ((16, 1), 576)))
    latent = d == 576
    dv = 512 if latent else d
    kv = rng.choice(("bf16", "bf16", "fp8") if latent else ("bf16", "bf16", "fp8", "f32"))
    page = rng.choice((16, 32, 64, 128, 256))
    hq, hkv = heads
    if op == "rope":
        tokens = _log(rng, 1, 32768)
        n = max(1, min(_log(rng, 1, 64), 40 * 32768 * 128 // (tokens * (hq + hkv) * d)))
        into, d = d, 64 if latent else d
        rot = rng.choice((d, d, d // 2, 24))
        start = rng.choice((0, d - rot))
        packed = tokens > 1 and rng.random() < 0.5
        return _rope(n=n, tokens=tokens, hq=hq, hkv=hkv, d=d, into=into, start=start, rot=rot, pairs=rng.random() < 0.5,
                     rule=rng.choice(("plain", "divide", "turns", "index")), base=rng.choice((10000.0, 500000.0)),
                     factor=rng.choice((2.0, 8.0, 40.0)), far=_log(rng, 1, 1 << 20), kv=rng.choice(("bf16", "f32")),
                     packed=packed, ragged=n > 1 and rng.random() < 0.5)
    row = hkv * (d + (0 if latent else dv)) * ELT[kv]
    if op == "append":
        tokens = _log(rng, 1, 32768)
        n = max(1, min(_log(rng, 1, 64), (512 << 20) // (tokens * row)))
        return _append(n=n, tokens=tokens, hkv=hkv, d=d, dv=dv, latent=latent, kv=kv, page=page,
                       held=_log(rng, 1, 5000), weighted=rng.random() < 0.5, packed=rng.random() < 0.5,
                       ragged=n > 1 and rng.random() < 0.5)
    rows = _log(rng, 1 if op == "decode" else 64, 131072)
    n = max(1, min(_log(rng, 1, 64), (768 << 20) // (rows * row)))
    if op == "decode":
        return _decode(n=n, rows=rows, hq=hq, hkv=hkv, d=d, dv=dv, latent=latent, kv=kv, page=page,
                       weigh=rng.random() < 0.5, ragged=n > 1 and rng.random() < 0.7)
    budget = _log(rng, 16, rows)
    sink, recent = rng.choice((0, 4)), max(1, budget // rng.choice((4, 8)))
    return _evict(n=n, rows=rows, hkv=hkv, d=d, dv=dv, latent=latent, kv=kv, page=page, sink=sink, recent=recent,
                  topk=max(0, budget - sink - recent), mixed=rng.random() < 0.5)


def lengths_of(n, longest, ragged):
    """The sequences' lengths: all the longest, or spread between one and it, the first the longest."""
    if not ragged:
        return [longest] * n
    return [max(1, int(longest * (1.0 - (b * 0.6180339887498949) % 1.0))) for b in range(n)]


# ---------------------------------------------------------------- what a program has in hand
def _rope_params(c):
    return dict(rot_start=c["start"], rot_dim=c["rot"], pairs=c["pairs"], rule=c["rule"], base=c["base"],
                factor=c["factor"], low_turns=1.0, high_turns=4.0 if c["rule"] == "turns" else 32.0, orig_len=8192,
                amplitude=1.25 if c["rule"] == "index" else 1.0)


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype)


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _slots(g, n):
    """n of n + 2 slots, in any order."""
    return torch.randperm(n + 2, generator=g, device=DEV)[:n]


def _pages(g, c, n, slots, lengths):
    """A page table over pages in random order, how many pages there are, and one that no sequence has; entries past a
    sequence's pages are -1."""
    counts = [-(-x // c["page"]) for x in lengths]
    n_pages = sum(counts) + 3
    perm = torch.randperm(n_pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((n + 2, max(counts)), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, m in zip(slots.tolist(), counts):
        table[s, :m] = perm[at:at + m]
        at += m
    return table, n_pages, perm[-1].long()


def _store(g, c, n_pages, width):
    shape = (n_pages, c["hkv"], c["page"], width)
    if c["kv"] != "fp8":
        return _randn(g, shape, KV_T[c["kv"]])
    x = torch.empty(shape, dtype=torch.uint8, device=DEV)
    for a in range(0, n_pages, 1024):  # codes of N(0, 1) values at a scale of 1 / 64
        x[a:a + 1024] = (_randn(g, tuple(x[a:a + 1024].shape), torch.float32) * 64).to(FP8).view(torch.uint8)
    return x


def _cache(g, c, n, slots, lengths):
    table, n_pages, spare = _pages(g, c, n, slots, lengths)
    s = dict(table=table, spare=spare, k=_store(g, c, n_pages, c["d"]), v=None if c["latent"] else _store(g, c, n_pages, c["dv"]))
    s["k_scale"] = s["v_scale"] = None
    if c["kv"] == "fp8":
        s["k_scale"] = (0.75 + 0.5 * torch.rand((n + 2, c["hkv"]), generator=g, device=DEV)) / 64
        s["v_scale"] = None if c["latent"] else (0.75 + 0.5 * torch.rand((n + 2, c["hkv"]), generator=g, device=DEV)) / 64
    s["token"] = torch.zeros((n_pages, c["hkv"], c["page"]), dtype=torch.int32, device=DEV)
    s["weight"] = torch.zeros((n_pages, c["hkv"], c["page"]), dtype=torch.float32, device=DEV)
    return s


def _heads(g, n, tokens, counts, dtype, packed):
    """[n, heads, tokens, d] for each (heads, d) of counts: views of one token-by-token buffer, or buffers of their own."""
    if not packed:
        return [_randn(g, (n, h, tokens, w), dtype) for h, w in counts]
    sizes = [h * w for h, w in counts]
    parts = _randn(g, (n, tokens, sum(sizes)), dtype).split(sizes, dim=-1)
    return [x.unflatten(-1, (h, w)).transpose(1, 2) for x, (h, w) in zip(parts, counts)]


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    n = c["n"]
    slots = _slots(g, n)
    s = dict(case=c, slots=slots, slot_ids=slots.to(torch.int32))
    if c["op"] == "rope":
        dtype = IN_T[c["kv"]]
        lengths = lengths_of(n, c["tokens"], c["ragged"])
        shapes = ((c["hq"], c["d"]), (c["hkv"], c["d"])) + (((c["hkv"], c["d"]),) if c["packed"] else ())
        s["q"], s["k"] = _heads(g, n, c["tokens"], shapes, dtype, c["packed"])[:2]
        s["pos"] = torch.randint(0, max(1, c["far"]), (n + 2,), generator=g, device=DEV, dtype=torch.int32)
        s["lengths"] = _i32(lengths) if c["ragged"] else None
        s["rope"] = _rope_params(c)
        s["q_out"], s["k_out"] = (torch.zeros(x.shape[:3] + (c["into"],), dtype=dtype, device=DEV) for x in (s["q"], s["k"]))
        s["live"] = torch.arange(c["tokens"], device=DEV)[None, :] < _i32(lengths)[:, None]
        return s
    dtype = IN_T[c["kv"]]
    if c["op"] == "append":
        lengths = lengths_of(n, c["tokens"], c["ragged"])
        held = [c["held"] * (b + 1) // n for b in range(n)]
        s.update(_cache(g, c, n, slots, [h + x for h, x in zip(held, lengths)]))
        s["rows"] = torch.zeros(n + 2, dtype=torch.int32, device=DEV)
        s["rows"][slots] = _i32(held)
        s["pos"] = s["rows"] + 100
        shapes = ((c["hkv"], c["d"]),) + (() if c["latent"] else ((c["hkv"], c["dv"]),))
        kv = _heads(g, n, c["tokens"], shapes, dtype, c["packed"])
        s["k_new"], s["v_new"] = kv[0], None if c["latent"] else kv[1]
        s["weight_new"] = torch.rand((n, c["hkv"], c["tokens"]), generator=g, device=DEV) if c["weighted"] else None
        s["lengths"] = _i32(lengths) if c["ragged"] else None
        s["b"] = torch.cat([torch.full((x,), b, device=DEV) for b, x in enumerate(lengths)])
        s["t"] = torch.cat([torch.arange(x, device=DEV) for x in lengths])
        return s
    if c["op"] == "decode":
        lengths = lengths_of(n, c["rows"], c["ragged"])
        s.update(_cache(g, c, n, slots, lengths))
        s["rows"] = torch.zeros(n + 2, dtype=torch.int32, device=DEV)
        s["rows"][slots] = _i32(lengths) - 1
        s["pos"] = s["rows"] + 77
        s["q"] = (2 * _randn(g, (n, c["hq"], c["d"]), torch.float32)).to(dtype)
        s["k_new"] = _randn(g, (n, c["hkv"], 1, c["d"]), dtype)
        s["v_new"] = None if c["latent"] else _randn(g, (n, c["hkv"], 1, c["dv"]), dtype)
        s["out"] = torch.zeros((n, c["hq"], c["dv"]), dtype=dtype, device=DEV)
        s["weight"].uniform_(0.0, 1.0, generator=g)
        s["weight0"] = s["weight"].clone() if c["weigh"] else None
        s["b"], s["t"] = torch.arange(n, device=DEV), torch.zeros(n, dtype=torch.long, device=DEV)
        return s
    rows = c["rows"]
    s.update(_cache(g, c, n, slots, [rows] * n))
    s["rows"] = torch.zeros(n + 2, dtype=torch.int32, device=DEV)
    s["rows"][slots] = rows
    s["rows_out"] = torch.zeros(n + 2, dtype=torch.int32, device=DEV)
    s["pos"] = torch.full((n + 2,), rows, dtype=torch.int32, device=DEV)
    per = s["table"].shape[1] * c["page"]
    token = torch.arange(per, device=DEV, dtype=torch.int32).expand(n, c["hkv"], per).clone()
    if c["mixed"]:  # the rows that an earlier eviction left are in no order, those stored since are
        m = min(rows, c["sink"] + c["recent"] + c["topk"])
        token[:, :, :m] = torch.rand((n, c["hkv"], m), generator=g, device=DEV).argsort(-1).to(torch.int32)
    weight = torch.exp(2 * _randn(g, (n, c["hkv"], per), torch.float32))
    weight = torch.where(torch.rand(weight.shape, generator=g, device=DEV) < 0.02, torch.zeros_like(weight), weight)
    pages = s["table"][slots].long().reshape(-1)
    for name, x in (("token", token), ("weight", weight)):
        s[name][pages] = x.unflatten(-1, (-1, c["page"])).transpose(1, 2).reshape(-1, c["hkv"], c["page"])
    s["token0"], s["weight0"] = s["token"].clone(), s["weight"].clone()
    s["kept"] = torch.zeros((n, c["hkv"], c["sink"] + c["recent"] + c["topk"]), dtype=torch.int32, device=DEV)
    return s


# ---------------------------------------------------------------- plain forms
def plain_frequencies(r):
    """Radians a position of every rotated pair (64 bits: far positions multiply them by up to 2^20)."""
    i = torch.arange(r["rot_dim"] // 2, dtype=torch.float64, device=DEV)
    f = torch.pow(torch.tensor(r["base"], dtype=torch.float64, device=DEV), -2.0 * i / r["rot_dim"])
    if r["rule"] == "plain":
        return f
    if r["rule"] == "divide":
        return f / r["factor"]
    if r["rule"] == "turns":  # between low and high turns over the original length, by the number of turns
        turns = r["orig_len"] * f / (2 * math.pi)
        keep = ((turns - r["low_turns"]) / (r["high_turns"] - r["low_turns"])).clamp(0.0, 1.0)
    else:  # by the index of the pair, between the indexes that make high and low turns
        at = lambda t: r["rot_dim"] * math.log(r["orig_len"] / (2 * math.pi * t)) / (2 * math.log(r["base"]))  # noqa: E731
        lo, hi = max(0.0, math.floor(at(r["high_turns"]))), min(r["rot_dim"] - 1.0, math.ceil(at(r["low_turns"])))
        keep = 1.0 - ((i - lo) / max(hi - lo, 0.001)).clamp(0.0, 1.0)
    return f / r["factor"] * (1.0 - keep) + f * keep


def plain_rope(x, r, positions):
    """x [n, heads, tokens, d] rotated at positions [n, tokens]."""
    angle = positions[:, None, :, None].double() * plain_frequencies(r)
    cos, sin = (angle.cos() * r["amplitude"]).float(), (angle.sin() * r["amplitude"]).float()
    a, m = r["rot_start"], r["rot_dim"]
    part = x[..., a:a + m].float()
    if r["pairs"]:
        x1, x2 = part[..., 0::2], part[..., 1::2]
        turned = torch.stack((x1 * cos - x2 * sin, x2 * cos + x1 * sin), dim=-1).flatten(-2)
    else:
        x1, x2 = part[..., :m // 2], part[..., m // 2:]
        turned = torch.cat((x1 * cos - x2 * sin, x2 * cos + x1 * sin), dim=-1)
    return torch.cat((x[..., :a], turned.to(x.dtype), x[..., a + m:]), dim=-1)


def plain_append(s, pages, new, scale):
    """new [n, hkv, tokens, d] into its rows of pages."""
    slot = s["slots"][s["b"]]
    row = s["rows"].long()[slot] + s["t"]
    x = new[s["b"], :, s["t"]]  # [live tokens, hkv, d]
    if pages.dtype == torch.uint8:
        x = (x.float() / scale[slot][..., None]).clamp(-448.0, 448.0).to(FP8).view(torch.uint8)
    page = pages.shape[2]
    pages[s["table"].long()[slot, row // page], :, row % page] = x


def plain_rows(s, pages, scale=None):
    """[n, hkv, rows, ...] of every slot's pages, in 32 bits; pages past a sequence's are page 0's."""
    x = pages[s["table"][s["slots"]].long().clamp(min=0)]  # [n, pages, hkv, page, ...]
    x = x.transpose(1, 2).flatten(2, 3)
    if x.dtype == torch.uint8:
        x = x.view(FP8).float() * scale[s["slots"]][:, :, None, None]
    return x


def plain_put(s, pages, rows, x):
    """x [n, hkv, m, ...] into rows [0, m) of every slot, where rows [n, 1, m] says so."""
    page, m = pages.shape[2], x.shape[2]
    at = torch.arange(m, device=DEV)
    p = s["table"][s["slots"]].long()[:, at // page]  # [n, m]
    p = torch.where(p < 0, s["spare"], p)  # not theirs: the unused page keeps what it holds
    old = pages[p, :, at % page].transpose(1, 2)
    keep = rows.reshape(rows.shape + (1,) * (x.dim() - 3))
    pages[p, :, at % page] = torch.where(keep, x, old).transpose(1, 2)


def plain_step(s):
    """The new token stored, and its attention over every row."""
    c = s["case"]
    plain_append(s, s["k"], s["k_new"], s["k_scale"])
    if s["v"] is not None:
        plain_append(s, s["v"], s["v_new"], s["v_scale"])
    slot = s["slots"]
    row, page = s["rows"].long()[slot], c["page"]
    at = s["table"].long()[slot, row // page], slice(None), row % page
    s["token"][at] = s["pos"][slot][:, None].expand(-1, c["hkv"])
    s["weight"][at] = 0.0
    k = plain_rows(s, s["k"], s["k_scale"]).float()
    v = k[..., :c["dv"]] if s["v"] is None else plain_rows(s, s["v"], s["v_scale"]).float()
    live = (torch.arange(k.shape[2], device=DEV)[None, :] <= row[:, None])[:, None, None, :]
    q = s["q"].float().unflatten(1, (c["hkv"], c["hq"] // c["hkv"]))
    z = (q @ k.transpose(-1, -2)) * (1.0 / math.sqrt(c["d"]))
    z = torch.where(live, z, torch.full_like(z, -math.inf))
    e = torch.exp(z - z.amax(-1, keepdim=True))
    p = e / e.sum(-1, keepdim=True)
    s["out"].copy_((p @ v).flatten(1, 2))
    if c["weigh"]:
        total = plain_rows(s, s["weight"]) + p.sum(2)
        plain_put(s, s["weight"], live[:, 0], total)


def plain_evict(s):
    c = s["case"]
    budget = c["sink"] + c["recent"] + c["topk"]
    held, pos = s["rows"][s["slots"]][:, None, None], s["pos"][s["slots"]][:, None, None]
    token, weight = plain_rows(s, s["token"]), plain_rows(s, s["weight"])
    at = torch.arange(token.shape[-1], device=DEV)
    live = at < held
    first = live & ((token < c["sink"]) | (token >= pos - c["recent"]))
    others = torch.where(live & ~first, weight, torch.full_like(weight, -1.0))
    order = others.sort(dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, at.expand_as(order).contiguous())
    keep = first | (live & ~first & (rank < budget - first.sum(-1, keepdim=True)))
    keep = torch.where(held > budget, keep, live)
    # the j-th kept row behind the budget goes to the j-th row before it that is not kept
    behind, hole = keep & (at >= budget), live & ~keep & (at < budget)
    far = token.shape[-1]
    source = torch.zeros(token.shape[:2] + (far + 1,), dtype=torch.long, device=DEV)
    source.scatter_(-1, torch.where(behind, behind.cumsum(-1) - 1, far), at.expand_as(token).contiguous())
    moved = source.gather(-1, (hole.cumsum(-1) - 1).clamp(min=0))
    kept = torch.where(hole, moved, at.expand_as(moved))[..., :budget]
    live = live[..., :budget].expand(kept.shape)
    s["kept"][..., :kept.shape[-1]] = torch.where(live, kept, -1).to(torch.int32)
    s["rows_out"][s["slots"]] = s["rows"][s["slots"]].clamp(max=budget)
    for name in ("k", "v", "token", "weight"):
        if s[name] is not None:
            x = s[name][s["table"][s["slots"]].long().clamp(min=0)].transpose(1, 2).flatten(2, 3)
            i = kept.reshape(kept.shape + (1,) * (x.dim() - 3)).expand(kept.shape + x.shape[3:])
            plain_put(s, s[name], live, x.gather(2, i))


def plain(s):
    c = s["case"]
    if c["op"] == "rope":
        positions = s["pos"][s["slots"]][:, None] + torch.arange(c["tokens"], device=DEV)
        for x, y in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
            y = y[..., c["into"] - c["d"]:]
            y.copy_(torch.where(s["live"][:, None, :, None], plain_rope(x, s["rope"], positions), y))
    elif c["op"] == "append":
        plain_append(s, s["k"], s["k_new"], s["k_scale"])
        if s["v"] is not None:
            plain_append(s, s["v"], s["v_new"], s["v_scale"])
        slot = s["slots"][s["b"]]
        row = s["rows"].long()[slot] + s["t"]
        at = s["table"].long()[slot, row // c["page"]], slice(None), row % c["page"]
        s["token"][at] = (s["pos"][slot] + s["t"].to(torch.int32))[:, None].expand(-1, c["hkv"])
        s["weight"][at] = 0.0 if s["weight_new"] is None else s["weight_new"][s["b"], :, s["t"]]
    elif c["op"] == "decode":
        plain_step(s)
    else:
        plain_evict(s)


# ---------------------------------------------------------------- the framework's calls
def _plan(s):
    """What the program sets up once: parameters, the cache's handle, a workspace."""
    import paper_2511_03092_amd as snap
    c = s["case"]
    code = {"f32": snap.SNAP_F32, "bf16": snap.SNAP_BF16, "fp8": snap.SNAP_FP8_E4M3}
    if c["op"] == "rope":
        rules = {"plain": snap.SNAP_ROPE_PLAIN, "divide": snap.SNAP_ROPE_DIVIDE, "turns": snap.SNAP_ROPE_BY_TURNS,
                 "index": snap.SNAP_ROPE_BY_INDEX}
        r = dict(s["rope"])
        r["layout"] = snap.SNAP_ROPE_PAIRS if r.pop("pairs") else snap.SNAP_ROPE_HALVES
        r["rule"] = rules[r["rule"]]
        return snap, snap.RopeParams(**r)
    p = snap.Params(n_q_heads=c.get("hq", c["hkv"]), n_kv_heads=c["hkv"], d_qk=c["d"], d_v=c["dv"],
                    sink=c.get("sink", 4), recent=c.get("recent", 64), topk=c.get("topk", 0), obs_window=1,
                    pool_kernel=1, v_in_k=c["latent"], in_dtype=code["f32" if c["kv"] == "f32" else "bf16"],
                    kv_dtype=code[c["kv"]])
    cache = snap.paged_cache_struct(s["k"], s["v"], s["table"], s["token"], s["weight"], s["k_scale"], s["v_scale"])
    ws = None
    if c["op"] == "decode":
        ws = snap.workspace(snap.snap_paged_decode_workspace(p, c["n"], c["rows"], c["weigh"]))
    elif c["op"] == "evict":
        ws = snap.workspace(snap.snap_paged_evict_workspace(p, c["n"], c["rows"]))
    return snap, p, cache, ws


def calls(s):
    c = s["case"]
    if "plan" not in s:
        s["plan"] = _plan(s)
    if c["op"] == "rope":
        snap, r = s["plan"]
        a = c["into"] - c["d"]
        snap.snap_rope(r, s["q"], s["k"], q_out=s["q_out"][..., a:], k_out=s["k_out"][..., a:], pos=s["pos"],
                       slot_ids=s["slot_ids"], lengths=s["lengths"])
        return
    snap, p, cache, ws = s["plan"]
    if c["op"] == "append":
        snap.snap_paged_append(p, cache, s["rows"], s["pos"], s["slot_ids"], s["k_new"], s["v_new"],
                               lengths=s["lengths"], weight_new=s["weight_new"])
    elif c["op"] == "decode":
        snap.snap_paged_decode_step(p, cache, s["rows"], s["pos"], s["slot_ids"], s["q"], s["k_new"], s["v_new"],
                                    s["out"], ws, max_rows=c["rows"], weigh=c["weigh"])
    else:
        snap.snap_paged_evict(p, cache, s["rows"], s["pos"], s["slot_ids"], s["rows_out"], ws, max_rows=c["rows"],
                              kept_out=s["kept"])


def run(state):
    s = state
    c = s["case"]
    # what the operator changes in place starts every pass from the same values
    if c["op"] == "decode" and c["weigh"]:
        s["weight"].copy_(s["weight0"])
    elif c["op"] == "evict":
        s["token"].copy_(s["token0"])
        s["weight"].copy_(s["weight0"])
    if own:
        calls(s)
    else:
        plain(s)
    if c["op"] == "rope":
        return dict(q=s["q_out"], k=s["k_out"])
    values = (lambda x: x.view(FP8)) if c["kv"] == "fp8" else (lambda x: x)
    got = dict(k=values(s["k"]), token=s["token"], weight=s["weight"])
    if s["v"] is not None:
        got["v"] = values(s["v"])
    if c["op"] == "decode":
        got["out"] = s["out"]
    elif c["op"] == "evict":
        got.update(kept=s["kept"], rows=s["rows_out"])
    return got


# ---------------------------------------------------------------- the work of a pass
def work(case):
    c = case
    if c["op"] == "rope":
        tokens = sum(lengths_of(c["n"], c["tokens"], c["ragged"]))
        elt = ELT["f32" if c["kv"] == "f32" else "bf16"]
        return dict(bytes=2 * tokens * (c["hq"] + c["hkv"]) * c["d"] * elt, flops=3 * tokens * (c["hq"] + c["hkv"]) * c["rot"])
    width = c["d"] + (0 if c["latent"] else c["dv"])
    row = c["hkv"] * width * ELT[c["kv"]]
    inrow = c["hkv"] * width * ELT["f32" if c["kv"] == "f32" else "bf16"]
    if c["op"] == "append":
        tokens = sum(lengths_of(c["n"], c["tokens"], c["ragged"]))
        return dict(bytes=tokens * (inrow + row + c["hkv"] * (12 if c["weighted"] else 8)), flops=0)
    if c["op"] == "decode":
        rows = sum(lengths_of(c["n"], c["rows"], c["ragged"]))
        io = c["n"] * c["hq"] * (c["d"] + c["dv"]) * ELT["f32" if c["kv"] == "f32" else "bf16"] + c["n"] * (inrow + row)
        return dict(bytes=rows * (row + (8 * c["hkv"] if c["weigh"] else 0)) + io,
                    flops=2 * rows * c["hq"] * (c["d"] + c["dv"]))
    budget = c["sink"] + c["recent"] + c["topk"]
    behind = max(0, c["rows"] - budget)
    late = min(c["recent"], behind)
    share = c["topk"] / max(1, c["rows"] - c["sink"] - c["recent"])
    moved = late + (behind - late) * min(1.0, share) if behind else 0
    return dict(bytes=c["n"] * (c["rows"] * 8 * c["hkv"] + moved * 2 * (row + 8 * c["hkv"]) + budget * 4 * c["hkv"]), flops=0)


# ---------------------------------------------------------------- from the definitions, in 64 bits
def _exact_rope(c, s):
    r = s["rope"]
    m, base = r["rot_dim"], r["base"]
    freq = []
    for j in range(m // 2):
        f = base ** (-2.0 * j / m)
        if r["rule"] == "divide":
            f /= r["factor"]
        elif r["rule"] == "turns":
            t = r["orig_len"] * f / (2 * math.pi)
            w = min(1.0, max(0.0, (t - r["low_turns"]) / (r["high_turns"] - r["low_turns"])))
            f = f * (w + (1.0 - w) / r["factor"])
        elif r["rule"] == "index":
            ends = [m * math.log(r["orig_len"] / (2 * math.pi * t)) / (2 * math.log(base)) for t in (r["high_turns"], r["low_turns"])]
            lo, hi = max(0, math.floor(ends[0])), min(m - 1, math.ceil(ends[1]))
            w = 1.0 - min(1.0, max(0.0, (j - lo) / max(hi - lo, 0.001)))
            f = f * (w + (1.0 - w) / r["factor"])
        freq.append(f)
    freq = torch.tensor(freq, dtype=torch.float64, device=DEV)
    lengths = lengths_of(c["n"], c["tokens"], c["ragged"])
    out = {}
    for name, before in (("q", s["q"]), ("k", s["k"])):
        y = s[name + "_out"].double()
        for b in range(c["n"]):
            x = before[b, :, :lengths[b]].double()
            start = int(s["pos"][int(s["slots"][b])])
            angle = (start + torch.arange(lengths[b], device=DEV, dtype=torch.float64))[:, None] * freq
            turn = torch.polar(torch.full_like(angle, r["amplitude"]), angle)
            part = x[..., r["rot_start"]:r["rot_start"] + m]
            z = torch.complex(part[..., 0::2].contiguous(), part[..., 1::2].contiguous()) if r["pairs"] else torch.complex(*part.chunk(2, -1))
            z = z * turn
            x[..., r["rot_start"]:r["rot_start"] + m] = (torch.view_as_real(z).flatten(-2) if r["pairs"] else torch.cat((z.real, z.imag), -1))
            y[b, :, :lengths[b], c["into"] - c["d"]:] = x
        out[name] = y
    return out


def _exact_store(s, c, lengths, pages, new, scale):
    """pages' values in 64 bits with the new tokens' in their rows (fp8: in units of the scale)."""
    if pages is None:
        return None
    y = (pages.view(FP8) if c["kv"] == "fp8" else pages).double()
    for b, x in enumerate(lengths):
        slot = int(s["slots"][b])
        first = int(s["rows"][slot])
        for a in range(0, x, 4096):
            row = first + torch.arange(a, min(x, a + 4096), device=DEV)
            value = new[b, :, a:min(x, a + 4096)].double()
            if c["kv"] == "fp8":
                value = (value / scale[slot].double()[:, None, None]).clamp(-448.0, 448.0)
            y[s["table"][slot, row // c["page"]].long(), :, row % c["page"]] = value.transpose(0, 1)
    return y


def _exact_decode(c, s):
    lengths = lengths_of(c["n"], c["rows"], c["ragged"])
    plain_append(s, s["k"], s["k_new"], s["k_scale"])  # the stored bits: attention is defined on them
    if s["v"] is not None:
        plain_append(s, s["v"], s["v_new"], s["v_scale"])
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    weight = s["weight"].double()
    group = c["hq"] // c["hkv"]
    for b, x in enumerate(lengths):
        slot = int(s["slots"][b])
        table = s["table"][slot, :-(-x // c["page"])].long()
        new = table[(x - 1) // c["page"]], slice(None), (x - 1) % c["page"]
        weight[new] = 0.0
        for h in range(c["hkv"]):
            def values(pages, scale):
                y = pages[table, h].flatten(0, 1)[:x]
                return y.double() if c["kv"] != "fp8" else y.view(FP8).double() * scale[slot, h].double()
            k = values(s["k"], s["k_scale"])
            v = k[:, :c["dv"]] if s["v"] is None else values(s["v"], s["v_scale"])
            p = torch.softmax(s["q"][b, h * group:(h + 1) * group].double() @ k.T.contiguous() / math.sqrt(c["d"]), -1)
            out[b, h * group:(h + 1) * group] = p @ v
            if c["weigh"]:
                row = torch.arange(x, device=DEV)
                weight[table[row // c["page"]], h, row % c["page"]] += p.sum(0)
    got = dict(k=None, token=None, weight=weight, out=out)
    if s["v"] is not None:
        got["v"] = None
    return got


def _exact_evict(c, s):
    budget, rows = c["sink"] + c["recent"] + c["topk"], c["rows"]
    got = {x: (s[x].view(FP8) if s[x].dtype == torch.uint8 else s[x]).double() for x in ("k", "v", "weight") if s[x] is not None}
    kept = np.full((c["n"], c["hkv"], budget), -1, dtype=np.int64)
    for b in range(c["n"]):
        table = s["table"][int(s["slots"][b])].long()
        token, weight = (s[x][table].transpose(0, 1).flatten(1).cpu().numpy()[:, :rows] for x in ("token", "weight"))
        for h in range(c["hkv"]):
            keep = np.arange(rows)
            if rows > budget:
                safe = (token[h] < c["sink"]) | (token[h] >= rows - c["recent"])
                other = np.flatnonzero(~safe)
                best = other[np.argsort(-weight[h][other].astype(np.float64), kind="stable")]
                keep = np.sort(np.concatenate((np.flatnonzero(safe), best[:budget - int(safe.sum())])))
            to = np.arange(len(keep))
            to[np.setdiff1d(to, keep, assume_unique=True)] = keep[keep >= len(keep)]
            kept[b, h, :len(to)] = to
            i = torch.from_numpy(to).to(DEV)
            j = torch.arange(len(to), device=DEV)
            for x in got.values():
                x[table[j // c["page"]], h, j % c["page"]] = x[table[i // c["page"]], h, i % c["page"]]
    got.update(token=None, kept=torch.from_numpy(kept).to(torch.int32), rows=None)
    return got


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "rope":
        return _exact_rope(c, s)
    if c["op"] == "decode":
        return _exact_decode(c, s)
    if c["op"] == "evict":
        return _exact_evict(c, s)
    lengths = lengths_of(c["n"], c["tokens"], c["ragged"])
    got = dict(k=_exact_store(s, c, lengths, s["k"], s["k_new"], s["k_scale"]), token=None)
    ones = torch.zeros((c["n"], c["hkv"], c["tokens"]), device=DEV) if s["weight_new"] is None else s["weight_new"]
    got["weight"] = _exact_store(s, dict(c, kv="f32"), lengths, s["weight"][..., None], ones[..., None], None)[..., 0]
    if s["v"] is not None:
        got["v"] = _exact_store(s, c, lengths, s["v"], s["v_new"], s["v_scale"])
    return got
