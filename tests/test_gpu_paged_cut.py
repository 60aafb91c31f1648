"""Attention over the paged cache where calls are cut into work items and joined (no call here is so short that a
workgroup takes a whole unit): pages that are not there, more than 64 sequences, and so many units that each is one item.
Against float64, with pagedhelp.attend's bounds, computed on the device.  Every case prints what names it before touching
the GPU."""
import math

import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import FP8, HALF_STEP, IN, P_ROUND, U, Paged, fill
from test_gpu_paged import SHAPES, _i32, _queries, _shape

pytestmark = pytest.mark.gpu


def _reference(c, slots, lengths, q):
    """Outputs [n, Hq, dv], their bounds, and the weights to add with theirs, in float64 on the device."""
    p = c.p
    G, scale = p.n_q_heads // p.n_kv_heads, 1.0 / math.sqrt(p.d_qk)
    out = torch.zeros((len(slots), p.n_q_heads, p.d_v), dtype=torch.float64, device="cuda")
    err, add, add_err = torch.zeros_like(out), torch.zeros(c.weight.shape, dtype=torch.float64, device="cuda"), None
    add_err = torch.zeros_like(add)
    for b, (s, n) in enumerate(zip(slots, lengths)):
        if n <= 0:
            continue
        r = torch.arange(n, device="cuda")
        page, off = c.table[s].long()[r // c.page], r % c.page
        there = (page >= 0) & (page < c.n_pages)
        page, off = page[there], off[there]
        if not len(page):
            continue

        def values(x, sc):
            y = x[page, :, off].transpose(0, 1)  # [h, rows, d]
            return (y.view(FP8).double() * sc[s].double()[:, None, None]) if c.kv == "fp8" else y.double()
        k = values(c.k, c.k_scale)
        v = k[..., :p.d_v] if p.v_in_k else values(c.v, c.v_scale)
        qb = q[b].double().view(p.n_kv_heads, G, p.d_qk)
        pr = torch.softmax(scale * torch.bmm(qb, k.transpose(1, 2).contiguous()), -1)
        dz = scale * (p.d_qk + 2) * U * torch.bmm(qb.abs(), k.abs().transpose(1, 2).contiguous()).amax(-1)  # [h, G]
        rel = 2 * dz + 80 * U
        out[b] = torch.bmm(pr, v).flatten(0, 1)
        err[b] = ((rel + P_ROUND[c.kv])[..., None] * torch.bmm(pr, v.abs())).flatten(0, 1)
        add[page, :, off] = pr.sum(1).T
        add_err[page, :, off] = (pr * rel[..., None]).sum(1).T
    return out, err, add, add_err


def _check(c, slots, lengths, q, out, before):
    want, err, add, add_err = _reference(c, slots, lengths, q)
    tol = HALF_STEP[out.dtype] * want.abs() * (1 + 2.0 ** -7) + err
    over = ((out.double() - want).abs() - tol).flatten(1).amax(1)
    assert bool((over <= 0).all()), (int(over.argmax()), lengths[int(over.argmax())], float(over.max()))
    if before is None:
        return
    total = before.double() + add
    same = torch.isnan(total) & torch.isnan(c.weight)
    assert bool((same | ((c.weight.double() - total).abs() <= add_err + 2 * U * total)).all())
    assert bool((same | (add > 0) | (c.weight == before)).all())


def _attend(c, slots, lengths, max_rows, weigh):
    p, n = c.p, len(slots)
    q = _queries(p, c.kv, n, 3)
    rows = c.rows.cpu()
    for s, x in zip(slots, lengths):
        rows[s] = x - 1
    c.rows.copy_(rows)
    out = torch.full((n, p.n_q_heads, p.d_v), 9.0, dtype=IN[c.kv], device="cuda")
    ws = snap.workspace(snap.snap_paged_decode_workspace(p, n, max_rows, weigh))
    ws.fill_(0xFF)
    before = c.weight.clone()
    snap.snap_paged_decode_attn(p, c.c, c.rows, _i32(slots), q, out, ws, max_rows=max_rows, weigh=weigh)
    torch.cuda.synchronize()
    if not weigh:
        assert torch.equal(torch.nan_to_num(before, -1.0), torch.nan_to_num(c.weight, -1.0))
    _check(c, slots, [min(x, max_rows) for x in lengths], q, out, before if weigh else None)


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("name", list(SHAPES))
def test_pages_that_are_not_there_in_calls_that_are_cut(name, weigh):
    """Items whose rows are all in missing pages, some of them, and none; sequences whose pages are all missing."""
    p, kv, page = _shape(name)
    lengths, max_rows = [2500, 700, 31, 1200, 64, 0], 1 << 15
    print(f"\n[case] paged decode {name}, missing pages, lengths {lengths} of at most {max_rows}, weigh {weigh}", flush=True)
    c = fill(Paged(p, kv, 6, page, lengths, 1, max_pages=max_rows // page), range(6), lengths, 2)
    table = c.table.cpu()
    for j in range(-(-2500 // page)):  # one page of three, and all of 512 rows together
        if j % 3 == 1 or 1024 <= j * page < 1536:
            table[0, j] = [-1, c.n_pages, -(1 << 31), 1 << 30][j % 4]
    table[1, :3] = -1
    table[3, :] = c.n_pages + 5
    table[4, 0] = -2
    c.table.copy_(table)
    _attend(c, list(range(6)), lengths, max_rows, weigh)


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("name", ["gqa-bf16", "g1-d64-bf16", "g16-bf16", "g3-fp8", "d64-fp8", "f32-d64", "f32-d128-g5",
                                  "keys-hold-values", "latent-bf16", "latent-fp8"])
@pytest.mark.parametrize("n", [65, 131])
def test_more_sequences_than_a_wave_has_lanes(name, n, weigh):
    """Sequences of nothing to 300 rows and a few long ones, one of which passes max_rows, in slots of any order."""
    p, kv, page = _shape(name)
    max_rows = 2500
    lengths = [(37 * b) % 300 for b in range(n)]
    lengths[3], lengths[63], lengths[64], lengths[n - 1] = 2500, 2100, 2600, 1025
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(n)).tolist()
    print(f"\n[case] paged decode {name}, {n} sequences of 0 to 2600 rows, weigh {weigh}", flush=True)
    cap = [0] * n
    for s, x in zip(slots, lengths):
        cap[s] = x
    c = fill(Paged(p, kv, n, page, cap, 1), slots, lengths, 2)
    _attend(c, slots, lengths, max_rows, weigh)


# as many units as make each one item, past the lengths that one workgroup takes
WHOLE = [("gqa-bf16", 514, 2100), ("d64-fp8", 2050, 2100), ("f32-d128-g5", 1030, 600), ("f32-d64", 2050, 1100),
         ("g3-fp8", 520, 4096), ("latent-bf16", 515, 4096), ("latent-fp8", 1030, 300)]


@pytest.mark.parametrize("weigh", [False, True])
@pytest.mark.parametrize("name,n,max_rows", WHOLE)
def test_units_that_are_an_item_each(name, n, max_rows, weigh):
    p, kv, page = _shape(name)
    lengths = [(7 * b) % 41 for b in range(n)]
    lengths[n // 2], lengths[n - 1] = max_rows, max_rows + 5
    print(f"\n[case] paged decode {name}, {n} sequences of 0 to 40 rows and two of {max_rows}, weigh {weigh}", flush=True)
    c = fill(Paged(p, kv, n, page, lengths, 1), range(n), lengths, 2)
    c.table[5 if lengths[5] else 6, 0] = -1
    _attend(c, list(range(n)), lengths, max_rows, weigh)


@pytest.mark.parametrize("name,n,max_rows", [("gqa-bf16", 514, 2100), ("g3-fp8", 131, 4096), ("f32-d128-g5", 1030, 600),
                                             ("latent-fp8", 131, 2000), ("d64-fp8", 1, 1 << 15)])
def test_steps_of_calls_that_are_cut(name, n, max_rows):
    """snap_paged_decode_step against the two calls, bit for bit: the new row at an item's start, inside and at its end."""
    p, kv, page = _shape(name)
    lengths = [(7 * b) % 67 for b in range(n)]
    lengths[n // 2] = max_rows - 40
    print(f"\n[case] paged step {name}, {n} sequences of 0 to 66 rows and one of {max_rows - 40}", flush=True)
    two = [fill(Paged(p, kv, n, page, [x + 1 for x in lengths], 1, max_pages=-(-max_rows // page)), range(n), lengths, 2) for _ in range(2)]
    g = torch.Generator().manual_seed(10)
    q, ids = _queries(p, kv, n, 20), _i32(list(range(n)))
    kn = torch.randn((n, p.n_kv_heads, 1, p.d_qk), generator=g).to(IN[kv]).cuda()
    vn = None if p.v_in_k else torch.randn((n, p.n_kv_heads, 1, p.d_v), generator=g).to(IN[kv]).cuda()
    ws = snap.workspace(snap.snap_paged_decode_workspace(p, n, max_rows, True))
    outs = [torch.empty((n, p.n_q_heads, p.d_v), dtype=IN[kv], device="cuda") for _ in range(2)]
    for c in two:
        c.rows.copy_(_i32(lengths))
        c.pos.copy_(_i32([x + 50 for x in lengths]))
    snap.snap_paged_decode_step(p, two[0].c, two[0].rows, two[0].pos, ids, q, kn, vn, outs[0], ws, max_rows=max_rows, weigh=True)
    snap.snap_paged_append(p, two[1].c, two[1].rows, two[1].pos, ids, kn, vn)
    before = two[1].weight.clone()
    snap.snap_paged_decode_attn(p, two[1].c, two[1].rows, ids, q, outs[1], ws, max_rows=max_rows, weigh=True)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    a, b = (c.state() for c in two)
    for x in ("k", "v", "token", "weight"):
        if a[x] is not None:
            assert torch.equal(a[x].view(torch.uint8), b[x].view(torch.uint8)), x
    _check(two[1], list(range(n)), [x + 1 for x in lengths], q, outs[1], before)


def test_debug_build_finds_no_more_items_than_are_launched():
    prev = snap.use_library(snap.DEBUG_LIB_PATH)
    try:
        snap.snap_debug_checks(reset=True)
        for name in ("gqa-bf16", "f32-d64", "latent-fp8"):
            test_more_sequences_than_a_wave_has_lanes(name, 65, True)
        test_units_that_are_an_item_each(*WHOLE[0], True)
        test_pages_that_are_not_there_in_calls_that_are_cut("g3-fp8", True)
        assert snap.snap_debug_checks(reset=True) == 0
    finally:
        snap._lib = prev
