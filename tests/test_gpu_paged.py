"""The paged cache against float64 on its own bytes: storing tokens, attention of one new token with and without
weights, eviction, and the four operators run together.  Unused rows and pages hold NaN, so a row read that is not held
shows.  Every case prints what names it before touching the GPU."""
import numpy as np
import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import FP8, HALF_STEP, IN, U, Paged, attend, evict, fill, params, rope

pytestmark = pytest.mark.gpu

# heads of q and k, width, values in the keys, type, page
SHAPES = {
    "gqa-bf16": (32, 8, 128, False, "bf16", 64),
    "g1-d64-bf16": (8, 8, 64, False, "bf16", 16),
    "g16-bf16": (16, 1, 128, False, "bf16", 32),
    "g3-fp8": (24, 8, 128, False, "fp8", 64),
    "d64-fp8": (16, 2, 64, False, "fp8", 16),
    "f32-d64": (4, 2, 64, False, "f32", 32),
    "f32-d128-g5": (10, 2, 128, False, "f32", 128),
    "keys-hold-values": (8, 2, 128, True, "bf16", 16),
    "f32-keys-hold-values": (4, 2, 64, True, "f32", 16),
    "latent-bf16": (8, 1, 576, True, "bf16", 64),
    "latent-g16-bf16": (16, 1, 576, True, "bf16", 16),
    "latent-fp8": (16, 1, 576, True, "fp8", 32),
    "latent-two-heads": (8, 2, 576, True, "bf16", 256),
}
RAGGED = [1, 300, 0, 31, 32, 33, 64, 17, 1000, 2, 129]


def _shape(name, **over):
    hq, hkv, d, latent, kv, page = SHAPES[name]
    return params(hq, hkv, d, kv, latent, **over), kv, page


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _queries(p, kv, n, seed):
    g = torch.Generator().manual_seed(seed)
    return (2 * torch.randn((n, p.n_q_heads, p.d_qk), generator=g)).to(IN[kv]).cuda()


def _check_decode(c, slots, lengths, q, out, before=None):
    """out (and the weights, when `before` is the state before the call) against float64."""
    p = c.p
    half = HALF_STEP[out.dtype]
    got = out.double().cpu().numpy()
    G = p.n_q_heads // p.n_kv_heads
    want_w = None if before is None else before["weight"].double().numpy().copy()
    tol_w = None if before is None else np.zeros_like(want_w)
    for b, (s, n) in enumerate(zip(slots, lengths)):
        o, err, pr, perr = attend(c, s, n, q[b])
        tol = half * np.abs(o) * (1 + 2.0 ** -7) + err
        assert (np.abs(got[b] - o) <= tol).all(), (b, n, float(np.abs(got[b] - o).max()), float(tol.max()))
        if before is not None:
            for r, (page, off) in enumerate(c.places(s, n)):
                if 0 <= page < c.n_pages:
                    for g in range(p.n_kv_heads):
                        want_w[page, g, off] += pr[g * G:(g + 1) * G, r].sum()
                        tol_w[page, g, off] = perr[g * G:(g + 1) * G, r].sum() + 2 * U * want_w[page, g, off]
    if before is not None:
        w = c.weight.double().cpu().numpy()
        same = np.isnan(want_w) & np.isnan(w)
        assert (same | (np.abs(w - want_w) <= tol_w)).all(), float(np.nanmax(np.abs(w - want_w) - tol_w))


def _decode(c, slots, lengths, seed, out_dtype, weigh, max_rows=None):
    n = len(slots)
    q = _queries(c.p, c.kv, n, seed)
    for s, x in zip(slots, lengths):
        c.rows[s] = x - 1
    out = torch.full((n, c.p.n_q_heads, c.p.d_v), 9.0, dtype=out_dtype, device="cuda")
    ml = max_rows or c.c.max_pages * c.c.page_size
    ws = snap.workspace(snap.snap_paged_decode_workspace(c.p, n, ml, weigh))
    ws.fill_(0xFF)
    before = c.state()
    snap.snap_paged_decode_attn(c.p, c.c, c.rows, _i32(slots), q, out, ws, max_rows=max_rows, weigh=weigh)
    torch.cuda.synchronize()
    return q, out, before


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("name", list(SHAPES))
def test_decode_of_ragged_sequences(name, weigh):
    p, kv, page = _shape(name)
    slots = [7, 3, 12, 0, 1, 5, 6, 10, 2, 11, 8]
    cap = [0] * 13
    for s, n in zip(slots, RAGGED):
        cap[s] = n
    print(f"\n[case] paged decode {name}, lengths {RAGGED}, weigh {weigh}", flush=True)
    c = fill(Paged(p, kv, 13, page, cap, 1), slots, RAGGED, 2)
    q, out, before = _decode(c, slots, RAGGED, 3, IN[kv], weigh)
    _check_decode(c, slots, RAGGED, q, out, before if weigh else None)
    after = c.state()
    for x in ("k", "v", "token") + (() if weigh else ("weight",)):
        if before[x] is not None:
            assert torch.equal(torch.nan_to_num(before[x].float()), torch.nan_to_num(after[x].float())), x


@pytest.mark.parametrize("name,n,length", [("gqa-bf16", 1, 9000), ("g3-fp8", 2, 5001), ("latent-bf16", 1, 6000),
                                           ("latent-fp8", 1, 4099), ("f32-d64", 1, 3001), ("g1-d64-bf16", 1, 7777),
                                           ("g16-bf16", 1, 384), ("g16-bf16", 1, 385), ("f32-d128-g5", 2, 128),
                                           ("f32-d128-g5", 1, 129), ("d64-fp8", 1, 768), ("d64-fp8", 1, 1025)])
@pytest.mark.parametrize("hint", [snap.SNAP_KV_STREAM, snap.SNAP_KV_KEEP])
def test_decode_of_long_sequences_split_over_the_card(name, n, length, hint):
    """Sequences cut into many items, and lengths around those that one workgroup takes whole."""
    p, kv, page = _shape(name, kv_reuse=hint)
    lengths = [length - 100 * b for b in range(n)]
    print(f"\n[case] paged decode {name}, lengths {lengths}, load hint {hint}", flush=True)
    c = fill(Paged(p, kv, n, page, lengths, 1), range(n), lengths, 2)
    q, out, before = _decode(c, list(range(n)), lengths, 3, torch.float32, True)
    _check_decode(c, list(range(n)), lengths, q, out, before)


@pytest.mark.parametrize("name,n", [("gqa-bf16", 300), ("latent-bf16", 300), ("f32-d64", 300), ("g3-fp8", 300),
                                    ("latent-bf16", 530), ("latent-fp8", 1030), ("latent-two-heads", 270)])
def test_decode_of_many_short_sequences(name, n):
    """More (sequence, KV head) units than work items are wanted, of 0 to 40 rows and one of 700."""
    p, kv, page = _shape(name)
    lengths = [(7 * b) % 41 for b in range(n)]
    lengths[n // 2] = 700
    print(f"\n[case] paged decode {name}, {n} sequences of 0 to 40 rows", flush=True)
    c = fill(Paged(p, kv, n, page, lengths, 1), range(n), lengths, 2)
    q, out, before = _decode(c, list(range(n)), lengths, 3, IN[kv], True)
    _check_decode(c, list(range(n)), lengths, q, out, before)


@pytest.mark.parametrize("name", ["gqa-bf16", "latent-bf16", "f32-d64", "latent-fp8", "g3-fp8", "keys-hold-values"])
def test_decode_with_pages_that_are_not_there_and_slots_out_of_range(name):
    """Rows in pages with ids out of range receive no attention (a sequence all of whose pages are missing gives
    zeros); rows past max_rows are not attended; sequences with bad slots leave their output alone."""
    p, kv, page = _shape(name)
    lengths = [5 * page + 3, 3 * page, 2 * page + 1, page // 2]
    print(f"\n[case] paged decode {name}, missing pages, lengths {lengths}", flush=True)
    c = Paged(p, kv, 6, page, lengths + [0, 0], 1)
    c.table[0, 1] = -1
    c.table[0, 4] = c.n_pages
    c.table[1, :] = 1 << 30
    c.table[2, 0] = -(1 << 31)
    fill(c, range(4), lengths, 2)
    limit = 4 * page + 1
    slots, held = [0, 1, 2, 3, -1, 6, 4], lengths + [0, 0, 0]
    q = _queries(p, kv, 7, 3)
    c.rows[:] = _i32([x - 1 for x in lengths] + [-1, 1 << 30])
    out = torch.full((7, p.n_q_heads, p.d_v), 9.0, dtype=torch.float32, device="cuda")
    ws = snap.workspace(snap.snap_paged_decode_workspace(p, 7, limit, True))
    before = c.state()
    snap.snap_paged_decode_attn(p, c.c, c.rows, _i32(slots), q, out, ws, max_rows=limit, weigh=True)
    torch.cuda.synchronize()
    assert bool((out[4:6] == 9.0).all()) and bool((out[1] == 0).all()) and bool((out[6] == 0).all())
    live = [0, 1, 2, 3]
    _check_decode(c, live, [min(x, limit) for x in lengths], q[:4], out[:4], before)
    assert held  # slot 4 holds no row


@pytest.mark.parametrize("name", list(SHAPES))
def test_step_is_append_then_attention(name):
    """snap_paged_decode_step against the two calls, bit for bit, over steps that cross pages; and against float64."""
    p, kv, page = _shape(name)
    lengths = [page - 2, 3 * page - 1, 0, 1]
    slots = [2, 0, 3, 4]
    cap = [0] * 5
    for s, x in zip(slots, lengths):
        cap[s] = x + 4
    print(f"\n[case] paged step {name}, rows {lengths}", flush=True)
    two = [fill(Paged(p, kv, 5, page, cap, 1), slots, lengths, 2) for _ in range(2)]
    for c in two:
        for s, x in zip(slots, lengths):
            c.rows[s], c.pos[s] = x, x + 50
    n, ids = len(slots), _i32(slots)
    ws = snap.workspace(snap.snap_paged_decode_workspace(p, n, two[0].c.max_pages * page, True))
    for step in range(3):
        g = torch.Generator().manual_seed(10 + step)
        q = _queries(p, kv, n, 20 + step)
        kn = torch.randn((n, p.n_kv_heads, 1, p.d_qk), generator=g).to(IN[kv]).cuda()
        vn = None if p.v_in_k else torch.randn((n, p.n_kv_heads, 1, p.d_v), generator=g).to(IN[kv]).cuda()
        outs = [torch.empty((n, p.n_q_heads, p.d_v), dtype=IN[kv], device="cuda") for _ in range(2)]
        snap.snap_paged_decode_step(p, two[0].c, two[0].rows, two[0].pos, ids, q, kn, vn, outs[0], ws, weigh=True)
        snap.snap_paged_append(p, two[1].c, two[1].rows, two[1].pos, ids, kn, vn)
        before = two[1].state()
        snap.snap_paged_decode_attn(p, two[1].c, two[1].rows, ids, q, outs[1], ws, weigh=True)
        torch.cuda.synchronize()
        a, b = (c.state() for c in two)
        for x in ("k", "v", "token", "weight"):
            if a[x] is not None:
                assert torch.equal(a[x].view(torch.uint8), b[x].view(torch.uint8)), (step, x)
        assert torch.equal(outs[0], outs[1]), step
        held = [x + step + 1 for x in lengths]
        _check_decode(two[1], slots, held, q, outs[1], before)
        for s, x in zip(slots, held):
            assert two[0].gather("token", s, 0, x)[0][-1] == x - 1 + 50
        for c in two:
            snap.snap_advance(c.rows, ids)
            snap.snap_advance(c.pos, ids)


@pytest.mark.parametrize("name", list(SHAPES))
@pytest.mark.parametrize("packed", [False, True])
def test_append_of_prompts(name, packed):
    """Ragged prompts behind rows already held, across pages and up to the end of the table, every byte compared; what
    was there stays."""
    p, kv, page = _shape(name)
    held, lengths, T = [0, page - 1, 3, 5, 2], [70, 33, 200, 1, 0], 90
    slots = [4, 0, 2, 1, 6]
    room = [2, 3, 4, 1, 1]  # pages
    cap = [0] * 6
    for s, m in zip(slots[:4], room):
        cap[s] = m * page
    print(f"\n[case] paged append {name}, held {held}, lengths {lengths} of {T}, packed {packed}", flush=True)
    c = Paged(p, kv, 6, page, cap, 1, max_pages=4)
    if c.table.shape[1] > 2:
        c.table[2, 1] = -5  # a page that is not there: its rows are dropped
    for s, h in zip(slots[:4], held):
        c.rows[s], c.pos[s] = h, h + 1000
    c.rows[5] = -1
    g = torch.Generator().manual_seed(5)
    n = len(slots)
    kn = torch.randn((n, p.n_kv_heads, T, p.d_qk), generator=g).to(IN[kv]) * 3
    vn = None if p.v_in_k else torch.randn((n, p.n_kv_heads, T, p.d_v), generator=g).to(IN[kv])
    wn = torch.rand((n, p.n_kv_heads, T), generator=g)
    wn[0, 0, 3], wn[0, 0, 4], wn[1, 0, 0] = float("nan"), float("inf"), -float("inf")
    before = c.state()
    dk, dvn = kn.cuda(), None if vn is None else vn.cuda()
    if packed:
        both = torch.cat([x.transpose(1, 2).flatten(2) for x in (kn, vn) if x is not None], -1).cuda()
        dk = both[..., :p.n_kv_heads * p.d_qk].unflatten(-1, (p.n_kv_heads, p.d_qk)).transpose(1, 2)
        dvn = None if vn is None else both[..., p.n_kv_heads * p.d_qk:].unflatten(-1, (p.n_kv_heads, p.d_v)).transpose(1, 2)
    snap.snap_paged_append(p, c.c, c.rows, c.pos, _i32(slots), dk, dvn, lengths=_i32(lengths), weight_new=wn.cuda())
    torch.cuda.synchronize()
    after, want = c.state(), before
    for b, s in enumerate(slots[:4]):
        n_new = min(lengths[b], T)
        total = min(held[b] + n_new, 4 * page)
        for r, (pg, off) in enumerate(c.places(s, total)):
            if r < held[b] or not 0 <= pg < c.n_pages:
                continue
            t = r - held[b]
            for x, new, sc in (("k", kn, c.k_scale), ("v", vn, c.v_scale)):
                if want[x] is None:
                    continue
                val = new[b, :, t]
                if kv == "fp8":
                    val = (val.float() / sc[s].cpu()[:, None]).clamp(-448, 448).to(FP8).view(torch.uint8)
                want[x][pg, :, off] = val
            want["token"][pg, :, off] = held[b] + 1000 + t
            w = wn[b, :, t].clone()
            w[~torch.isfinite(w)] = 0
            want["weight"][pg, :, off] = w
    for x in ("k", "v", "token", "weight", "rows", "pos"):
        if want[x] is not None:
            assert torch.equal(want[x].view(torch.uint8), after[x].view(torch.uint8)), x


def _evict_case(p, kv, page, slots, rows, pos, tokens, weights, max_rows=None, n_slots=None, table_rows=0):
    """Runs an eviction over given tokens and weights [sequence][head][row] and checks every byte.  table_rows: the page
    table has room for so many, and so the call for as many rows."""
    n, B, h = len(slots), p.budget, p.n_kv_heads
    n_slots = n_slots or max(slots) + 1
    cap = [0] * n_slots
    for s, r in zip(slots, rows):
        cap[s] = r
    c = fill(Paged(p, kv, n_slots, page, cap, 1, max_pages=table_rows // page or None), slots, rows, 2)
    st = c.state()
    for b, s in enumerate(slots):
        c.rows[s], c.pos[s] = rows[b], pos[b]
        pg, off = (torch.tensor(x, dtype=torch.long) for x in zip(*c.places(s, rows[b]) or [(0, 0)]))
        for g in range(h if rows[b] else 0):
            st["token"][pg, g, off] = torch.as_tensor(np.asarray(tokens[b][g]).astype(np.int32))
            st["weight"][pg, g, off] = torch.as_tensor(np.asarray(weights[b][g]).astype(np.float32))
    c.token.copy_(st["token"])
    c.weight.copy_(st["weight"])
    out = torch.full((n_slots,), -3, dtype=torch.int32, device="cuda")
    kept = torch.full((n, h, B), -9, dtype=torch.int32, device="cuda")
    ml = max_rows or c.c.max_pages * page
    ws = snap.workspace(snap.snap_paged_evict_workspace(p, n, ml))
    ws.fill_(0xFF)
    before = c.state()
    snap.snap_paged_evict(p, c.c, c.rows, c.pos, _i32(slots), out, ws, max_rows=max_rows, kept_out=kept)
    torch.cuda.synchronize()
    after, want = c.state(), {x: (None if v is None else v.clone()) for x, v in before.items()}
    got = kept.cpu().numpy()
    for b, s in enumerate(slots):
        R = min(rows[b], ml)
        assert int(out[s]) == min(R, B)
        pl = c.places(s, rows[b])
        for g in range(h):
            w = np.float32(weights[b][g][:R])
            exp = evict(np.asarray(tokens[b][g][:R]), w, R, pos[b], p.sink, p.recent, B)
            assert np.array_equal(got[b, g], exp), (b, g, np.flatnonzero(got[b, g] != exp)[:5])
            to = np.flatnonzero((exp >= 0) & (exp != np.arange(B)))
            if len(to):
                (tp, to_), (fp, fo) = ((torch.tensor(x, dtype=torch.long) for x in zip(*[pl[i] for i in idx]))
                                       for idx in (to, exp[to]))
                for x in ("k", "v", "token", "weight"):
                    if want[x] is not None:
                        want[x][tp, g, to_] = before[x][fp, g, fo]
    for x in ("k", "v", "token", "weight", "rows", "pos"):
        if want[x] is not None:
            assert torch.equal(want[x].contiguous().view(torch.uint8), after[x].contiguous().view(torch.uint8)), x
    others = [s for s in range(n_slots) if s not in slots]
    assert all(int(out[s]) == -3 for s in others)
    return c


# the calls' most rows: what one workgroup selects among, and more (the rows held are the same)
@pytest.mark.parametrize("table_rows", [0, 1 << 14])
@pytest.mark.parametrize("name", list(SHAPES))
def test_evict_ragged(name, table_rows):
    """Slots above, at and below the budget, tokens in any order, weights with many ties."""
    p, kv, page = _shape(name, sink=3, recent=9, topk=40)
    rows = [200, 52, 53, 7, 0, 97, 1030]
    slots = [6, 1, 2, 8, 0, 4, 3]
    rng = np.random.default_rng(3)
    pos = [r + 30 for r in rows]
    tokens = [[rng.permutation(r + 30)[:r] for _ in range(p.n_kv_heads)] for r in rows]
    weights = [[np.round(rng.exponential(1.0, r) * 4) / 4 for _ in range(p.n_kv_heads)] for r in rows]
    print(f"\n[case] evict {name}, rows {rows}, budget {p.budget}", flush=True)
    _evict_case(p, kv, page, slots, rows, pos, tokens, weights, n_slots=9, table_rows=table_rows)


@pytest.mark.parametrize("table_rows", [0, 9000 // 32 * 32, 1 << 18])
@pytest.mark.parametrize("what", ["all-equal", "zeros", "nan-and-negative", "huge-and-tiny", "ascending", "no-topk",
                                  "no-sink", "all-protected", "one-row-over", "max-rows"])
def test_evict_edges(what, table_rows):
    over = dict(sink=2, recent=5, topk=30)
    rows, max_rows = 300, None
    if what == "no-topk":
        over["topk"] = 0
    elif what == "no-sink":
        over["sink"] = 0
    p, kv, page = _shape("f32-d64", **over)
    if what == "one-row-over":
        rows = p.budget + 1
    if what == "max-rows":
        max_rows = 77
    rng = np.random.default_rng(7)
    tok = [[np.arange(rows) for _ in range(2)]]
    w = rng.exponential(1.0, (2, rows)).astype(np.float32)
    if what == "all-equal":
        w[:] = 0.25
    elif what == "zeros":
        w[:, 20:] = 0
    elif what == "nan-and-negative":
        w[:, ::3], w[:, 1::3] = np.nan, -w[:, 1::3]
    elif what == "huge-and-tiny":
        w[0, ::2], w[1, ::2] = np.inf, 3e38
        w[:, 1::2] = 1e-42  # subnormal
    elif what == "ascending":
        w[:] = np.arange(rows)
    elif what == "all-protected":
        tok = [[np.zeros(rows, int) for _ in range(2)]]
    print(f"\n[case] evict {what}", flush=True)
    _evict_case(p, kv, page, [0], [rows], [rows], tok, [w], max_rows=max_rows, table_rows=table_rows)


@pytest.mark.parametrize("topk", [0, 1, 2, 3, 4091, 4092, 4093, 4094, 4095, 8190, 8999])
def test_evict_to_budgets_around_the_splits(topk):
    """Budgets at every remainder of 4 and around whole tiles, rows that end inside one; weights with ties, so that the
    rows of the last weight kept lie on both sides of the budget."""
    p, kv, page = _shape("f32-d64", sink=0, recent=1, topk=topk)
    rng = np.random.default_rng(topk)
    rows = [9003, topk + 2, 8193]
    print(f"\n[case] evict {rows} rows to {p.budget}", flush=True)
    _evict_case(p, kv, page, [1, 0, 2], rows, rows, [[rng.permutation(r) for _ in range(2)] for r in rows],
                [np.round(rng.exponential(1.0, (2, r)) * 2).astype(np.float32) for r in rows])


def test_evict_of_a_long_sequence():
    """Many splits, and splits of several tiles; most rows evicted, and most kept."""
    rng = np.random.default_rng(11)
    for rows, topk in ((40001, 500), (36007, 33000), (150001, 70003)):
        p = params(4, 2, 64, "bf16", sink=4, recent=100, topk=topk)
        print(f"\n[case] evict {rows} rows to {p.budget}", flush=True)
        _evict_case(p, "bf16", 256, [0], [rows], [rows], [[rng.permutation(rows) for _ in range(2)]],
                    [rng.exponential(1.0, (2, rows)).astype(np.float32) ** 4])


def test_prompt_steps_and_evictions_together():
    """A program's use of all of them: prompts rotated out of the packed projection and stored, steps that weigh,
    evictions whenever a slot outgrows its budget, counters moved by snap_advance; a mirror in float64 follows.  Twice
    over, eagerly and with every step captured as a graph: the same bits."""
    p = params(8, 2, 64, "bf16", sink=2, recent=12, topk=34)
    r = snap.RopeParams(0, 64, base=500000.0)
    page, lengths, slots, n_slots, T = 16, [60, 37], [2, 0], 3, 60
    cap = [6 * page, 0, 6 * page]
    results = []
    for graphed in (False, True):
        print(f"\n[case] rotary, paged steps and evictions, graph {graphed}", flush=True)
        g = torch.Generator().manual_seed(8)
        c = Paged(p, "bf16", n_slots, page, cap, 1)
        c.weight.zero_()
        ids, H = _i32(slots), p.n_q_heads + 2 * p.n_kv_heads
        x = torch.randn((2, T, H, 64), generator=g).bfloat16().cuda()
        heads = x.transpose(1, 2)
        q, k, v = heads[:, :8], heads[:, 8:10], heads[:, 10:]
        kr = torch.empty(k.shape, dtype=k.dtype, device="cuda")
        qr = torch.empty(q.shape, dtype=q.dtype, device="cuda")
        snap.snap_rope(r, q, k, qr, kr)
        snap.snap_paged_append(p, c.c, c.rows, c.pos, ids, kr, v, lengths=_i32(lengths))
        c.rows[ids.long()] += _i32(lengths)
        c.pos[ids.long()] += _i32(lengths)
        ml = 6 * page
        ws = snap.workspace(max(snap.snap_paged_decode_workspace(p, 2, ml, True), snap.snap_paged_evict_workspace(p, 2, ml)))
        rows_out = torch.zeros(n_slots, dtype=torch.int32, device="cuda")
        kept = torch.empty((2, p.n_kv_heads, p.budget), dtype=torch.int32, device="cuda")
        step = torch.zeros((2, 1, H, 64), dtype=torch.bfloat16, device="cuda")
        sq, sk = (torch.empty((2, h, 1, 64), dtype=torch.bfloat16, device="cuda") for h in (8, 2))
        out = torch.empty((2, 8, 64), dtype=torch.bfloat16, device="cuda")

        def one_step():
            hs = step.transpose(1, 2)
            snap.snap_rope(r, hs[:, :8], hs[:, 8:10], sq, sk, pos=c.pos, slot_ids=ids)
            vn = hs[:, 10:].contiguous()
            snap.snap_paged_decode_step(p, c.c, c.rows, c.pos, ids, sq.view(2, 8, 64), sk, vn, out, ws, weigh=True)
            snap.snap_advance(c.rows, ids)
            snap.snap_advance(c.pos, ids)

        graph = None
        if graphed:
            keep = {t: getattr(c, t).clone() for t in ("k", "v", "token", "weight", "rows", "pos")}
            one_step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                one_step()
            for t, val in keep.items():
                getattr(c, t).copy_(val)
        log = []
        for i in range(45):
            fresh = torch.randn((2, 1, H, 64), generator=g).bfloat16()
            step.copy_(fresh.cuda())
            before = c.state()
            graph.replay() if graphed else one_step()
            torch.cuda.synchronize()
            held = [int(before["rows"][s]) + 1 for s in slots]
            st = c.state()
            for b, s in enumerate(slots):  # the new key is the rotated one, at its position
                pg, off = c.places(s, held[b])[-1]
                want, size = rope(r, fresh[b, 0, 8:10].double().numpy(), np.full(2, float(before["pos"][s])))
                err = np.abs(st["k"][pg, :, off].double().numpy() - want)
                assert (err <= 2.0 ** -8 * np.abs(want) * 1.01 + 8 * U * size).all()
                assert bool((st["token"][pg, :, off] == before["pos"][s]).all())
                before["weight"][pg, :, off] = 0
            if not graphed:
                _check_decode(c, slots, held, sq.view(2, 8, 64), out, before)
            log.append(out.clone())
            if i % 11 == 10:
                b4 = c.state()
                snap.snap_paged_evict(p, c.c, c.rows, c.pos, ids, rows_out, ws, max_rows=ml, kept_out=kept)
                torch.cuda.synchronize()
                for b, s in enumerate(slots):
                    R = int(b4["rows"][s])
                    for h in range(2):
                        tok, w = (c.gather(t, s, h, R, b4)[0].numpy() for t in ("token", "weight"))
                        exp = evict(tok, w, R, int(b4["pos"][s]), p.sink, p.recent, p.budget)
                        assert np.array_equal(kept[b, h].cpu().numpy(), exp)
                        now = c.gather("token", s, h, min(R, p.budget))[0].numpy()
                        assert set(range(p.sink)) <= set(now.tolist())
                        assert set(range(int(b4["pos"][s]) - p.recent, int(b4["pos"][s]))) <= set(now.tolist())
                c.rows.copy_(torch.where(torch.isin(torch.arange(n_slots, device="cuda"), ids.long()), rows_out, c.rows))
        results.append((torch.stack(log).cpu(), c.state()))
    (la, sa), (lb, sb) = results
    assert torch.equal(la, lb)
    for x in ("k", "v", "token", "weight", "rows", "pos"):
        assert torch.equal(sa[x].contiguous().view(torch.uint8), sb[x].contiguous().view(torch.uint8)), x


def test_prompt_scores_as_first_weights_select_what_compression_selects():
    """snap_compress's pooled scores as the prompt's weights: cutting the paged prompt to the same budget keeps the
    tokens that compression keeps."""
    p = params(8, 2, 64, "bf16", sink=4, recent=64, topk=200, obs_window=16, pool_kernel=7)
    L, page = 1500, 64
    print("\n[case] pooled scores as first weights", flush=True)
    g = torch.Generator().manual_seed(4)
    q = torch.randn((1, 8, 16, 64), generator=g).bfloat16().cuda()
    k, v = (torch.randn((1, 2, L, 64), generator=g).bfloat16().cuda() for _ in range(2))
    ck, cv = (torch.zeros((1, 2, p.budget, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    zero, len_ = _i32([0]), _i32([L])
    pos, ntop = _i32([0]), _i32([0])
    sel = torch.empty((1, 2, p.topk), dtype=torch.int32, device="cuda")
    pooled = torch.empty((1, 2, L), dtype=torch.float32, device="cuda")
    snap.snap_compress(p, snap.cache_struct(ck, cv), pos, ntop, zero, len_, q, k, v,
                       snap.workspace(snap.snap_compress_workspace(p, 1, L)), sel_out=sel, pooled_out=pooled)
    c = Paged(p, "bf16", 1, page, [L], 1)
    snap.snap_paged_append(p, c.c, c.rows, c.pos, zero, k, v, weight_new=pooled)
    c.rows += L
    c.pos += L
    kept = torch.empty((1, 2, p.budget), dtype=torch.int32, device="cuda")
    out = torch.zeros_like(c.rows)
    snap.snap_paged_evict(p, c.c, c.rows, c.pos, zero, out, snap.workspace(snap.snap_paged_evict_workspace(p, 1, L)),
                          max_rows=L, kept_out=kept)
    torch.cuda.synchronize()
    for h in range(2):
        want = set(range(p.sink)) | set(range(L - p.recent, L)) | set(sel[0, h].cpu().tolist())
        assert set(kept[0, h].cpu().tolist()) == want
        assert set(c.gather("token", 0, h, p.budget)[0].tolist()) == want
    assert int(out[0]) == p.budget


def test_two_streams_on_their_own_caches():
    """Calls on two streams at once, each with its own cache and workspace: the bits of the calls one after the other."""
    p, kv, page = _shape("gqa-bf16")
    print("\n[case] paged decode on two streams", flush=True)
    lengths = [900, 1500]
    cs = [fill(Paged(p, kv, 1, page, [n], 1), [0], [n], 2 + i) for i, n in enumerate(lengths)]
    want = []
    for c, n in zip(cs, lengths):
        q, out, before = _decode(c, [0], [n], 3, torch.bfloat16, True)
        want.append((out.clone(), c.weight.clone()))
        c.weight.copy_(before["weight"])
    streams = [torch.cuda.Stream() for _ in cs]
    outs = [torch.empty_like(w[0]) for w in want]
    qs = [_queries(p, kv, 1, 3) for _ in cs]
    wss = [snap.workspace(snap.snap_paged_decode_workspace(p, 1, c.c.max_pages * page, True)) for c in cs]
    ids = _i32([0])
    torch.cuda.synchronize()
    for c, st, q, o, ws in zip(cs, streams, qs, outs, wss):
        with torch.cuda.stream(st):
            snap.snap_paged_decode_attn(p, c.c, c.rows, ids, q, o, ws, weigh=True)
    torch.cuda.synchronize()
    for c, o, w in zip(cs, outs, want):
        assert torch.equal(o, w[0])
        assert torch.equal(torch.nan_to_num(c.weight), torch.nan_to_num(w[1]))


@pytest.mark.parametrize("name,length", [("gqa-bf16", 60), ("gqa-bf16", 3000), ("f32-d64", 2500), ("d64-fp8", 2500),
                                         ("latent-bf16", 700), ("latent-fp8", 700)])
def test_captured_steps_replay(name, length):
    """A step with weights captured once and replayed, the counters moving inside the graph, beside eager steps of a twin
    cache that shares the workspace: the same bits after every replay."""
    p, kv, page = _shape(name)
    lengths, slots = [length, length // 3], [1, 0]
    print(f"\n[case] captured paged step {name}, rows {lengths}", flush=True)
    cap = [length // 3 + 8, length + 8]
    two = [fill(Paged(p, kv, 2, page, cap, 1), slots, lengths, 2) for _ in range(2)]
    for c in two:
        for s, x in zip(slots, lengths):
            c.rows[s], c.pos[s] = x, x + 9
    ids, ml = _i32(slots), two[0].c.max_pages * page
    ws = snap.workspace(snap.snap_paged_decode_workspace(p, 2, ml, True))
    g = torch.Generator().manual_seed(6)
    q = _queries(p, kv, 2, 7)
    kn = torch.randn((2, p.n_kv_heads, 1, p.d_qk), generator=g).to(IN[kv]).cuda()
    vn = None if p.v_in_k else torch.randn((2, p.n_kv_heads, 1, p.d_v), generator=g).to(IN[kv]).cuda()
    outs = [torch.empty((2, p.n_q_heads, p.d_v), dtype=IN[kv], device="cuda") for _ in range(2)]

    def step(i):
        c = two[i]
        snap.snap_paged_decode_step(p, c.c, c.rows, c.pos, ids, q, kn, vn, outs[i], ws, weigh=True)
        snap.snap_advance(c.rows, ids)
        snap.snap_advance(c.pos, ids)

    step(0)
    step(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for i in range(4):
        q.copy_(_queries(p, kv, 2, 30 + i))
        graph.replay()
        torch.cuda.synchronize()
        step(1)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]), i
        a, b = (c.state() for c in two)
        for x in ("k", "v", "token", "weight", "rows", "pos"):
            if a[x] is not None:
                assert torch.equal(a[x].view(torch.uint8), b[x].view(torch.uint8)), (i, x)


@pytest.mark.parametrize("name", ["gqa-bf16", "f32-d64", "latent-fp8", "latent-bf16"])
@pytest.mark.parametrize("bound", [40, 2000])
def test_step_past_max_rows_stores_the_token_without_attending_it(name, bound):
    p, kv, page = _shape(name)
    held = bound + 7
    print(f"\n[case] paged step {name}, {held} rows of which {bound} are attended", flush=True)
    c = fill(Paged(p, kv, 1, page, [held + 1], 1), [0], [held], 2)
    c.rows[0], c.pos[0] = held, 500
    before = c.state()
    g = torch.Generator().manual_seed(5)
    kn = torch.randn((1, p.n_kv_heads, p.d_qk), generator=g).to(IN[kv]).cuda()
    vn = None if p.v_in_k else torch.randn((1, p.n_kv_heads, p.d_v), generator=g).to(IN[kv]).cuda()
    q = _queries(p, kv, 1, 7)
    out = torch.empty((1, p.n_q_heads, p.d_v), dtype=IN[kv], device="cuda")
    snap.snap_paged_decode_step(p, c.c, c.rows, c.pos, _i32([0]), q, kn, vn, out,
                                snap.workspace(snap.snap_paged_decode_workspace(p, 1, bound, True)), max_rows=bound,
                                weigh=True)
    torch.cuda.synchronize()
    pg, off = c.places(0, held + 1)[-1]
    before["weight"][pg, :, off] = 0
    _check_decode(c, [0], [bound], q, out, before)
    assert bool((c.token[pg, :, off] == 500).all())
    if kv != "fp8":
        assert torch.equal(c.k[pg, :, off], kn[0])


@pytest.mark.parametrize("name,pages", [("gqa-bf16", 40000), ("latent-bf16", 60000)])
def test_pages_past_four_gigabytes(name, pages):
    """Pages whose elements lie past 2^31 and whose bytes past 2^32, through all four calls."""
    p, kv, page = _shape(name, sink=2, recent=20, topk=100)
    print(f"\n[case] paged calls {name}, {pages} pages of {page} rows", flush=True)
    h, length, dev = p.n_kv_heads, 300, "cuda"
    small = fill(Paged(p, kv, 1, page, [length + 1], 1), [0], [length], 2)
    big = Paged.__new__(Paged)
    big.p, big.kv, big.page, big.n_slots, big.n_pages, big.max_pages = p, kv, page, 1, pages, small.max_pages
    big.k_scale = big.v_scale = None
    big.k = torch.empty((pages, h, page, p.d_qk), dtype=torch.bfloat16, device=dev)
    big.v = None if p.v_in_k else torch.empty((pages, h, page, p.d_v), dtype=torch.bfloat16, device=dev)
    big.token = torch.zeros((pages, h, page), dtype=torch.int32, device=dev)
    big.weight = torch.zeros((pages, h, page), device=dev)
    assert big.k.numel() > 1 << 31
    n = small.max_pages
    ids = [pages - 1 - 3 * j for j in range(n)]
    big.table = torch.tensor([ids], dtype=torch.int32, device=dev)
    for x in ("k", "v", "token", "weight"):
        if getattr(big, x) is not None:
            getattr(big, x)[ids] = getattr(small, x)[small.table[0].long()]
    big.rows, big.pos = small.rows.clone(), small.pos.clone()
    big.handle()
    ids = _i32([0])
    g = torch.Generator().manual_seed(5)
    kn = torch.randn((1, h, 1, p.d_qk), generator=g).to(IN[kv]).cuda()
    vn = None if p.v_in_k else torch.randn((1, h, 1, p.d_v), generator=g).to(IN[kv]).cuda()
    q, ml = _queries(p, kv, 1, 7), n * page
    got = []
    for c in (small, big):
        c.rows[0] = c.pos[0] = length
        ws = snap.workspace(max(snap.snap_paged_decode_workspace(p, 1, ml, True), snap.snap_paged_evict_workspace(p, 1, ml)))
        out = torch.empty((1, p.n_q_heads, p.d_v), dtype=IN[kv], device=dev)
        snap.snap_paged_append(p, c.c, c.rows, c.pos, ids, kn, vn)
        snap.snap_paged_decode_step(p, c.c, c.rows, c.pos, ids, q, kn, vn, out, ws, weigh=True)
        snap.snap_advance(c.rows, ids)
        snap.snap_advance(c.pos, ids)
        rows_out = torch.zeros_like(c.rows)
        kept = torch.empty((1, h, p.budget), dtype=torch.int32, device=dev)
        snap.snap_paged_evict(p, c.c, c.rows, c.pos, ids, rows_out, ws, kept_out=kept)
        torch.cuda.synchronize()
        pg = c.table[0].long()
        got.append([out, kept] + [getattr(c, x)[pg] for x in ("k", "v", "token", "weight") if getattr(c, x) is not None])
    for a, b in zip(*got):
        assert torch.equal(torch.nan_to_num(a.float()), torch.nan_to_num(b.float()))


@pytest.fixture
def debug_library():
    prev = snap.use_library(snap.DEBUG_LIB_PATH)
    try:
        snap.snap_debug_checks(reset=True)
        yield
    finally:
        snap._lib = prev


def test_debug_build_records_no_failed_invariant_of_the_paged_calls(debug_library):
    for name in ("gqa-bf16", "g3-fp8", "f32-d64", "latent-bf16", "latent-fp8"):
        test_decode_of_ragged_sequences(name, True)
        test_step_is_append_then_attention(name)
        test_evict_ragged(name, 0)
        test_evict_ragged(name, 1 << 14)
        assert snap.snap_debug_checks(reset=True) == 0, name
