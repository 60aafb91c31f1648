"""Eviction where its bounds meet: counters below zero, calls whose max_rows is less than the rows held, on both selection
paths.  Every byte of the cache is compared.  Every case prints what names it before touching the GPU."""
import numpy as np
import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import Paged, evict, fill, params

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _run(p, kv, page, cap, rows, max_rows, seed=0, before=None):
    """Slot i holds rows[i] rows (a page table with room for cap[i]); the cache, its state before and the call's outputs.
    before(cache): changes to it first."""
    n = len(rows)
    c = fill(Paged(p, kv, n, page, cap, 1), range(n), [max(0, min(r, x)) for r, x in zip(rows, cap)], 2 + seed)
    c.rows.copy_(_i32(rows))
    c.pos.copy_(_i32([max(0, r) + 30 for r in rows]))
    if before:
        before(c)
    out = torch.full((n,), -3, dtype=torch.int32, device="cuda")
    kept = torch.full((n, p.n_kv_heads, p.budget), -9, dtype=torch.int32, device="cuda")
    ws = snap.workspace(snap.snap_paged_evict_workspace(p, n, max_rows))
    ws.fill_(0xFF)
    state = c.state()
    snap.snap_paged_evict(p, c.c, c.rows, c.pos, _i32(list(range(n))), out, ws, max_rows=max_rows, kept_out=kept)
    torch.cuda.synchronize()
    return c, state, out.tolist(), kept.cpu().numpy()


def _same(a, b):
    for x in ("k", "v", "token", "weight", "rows", "pos"):
        if a[x] is not None:
            assert torch.equal(a[x].contiguous().view(torch.uint8), b[x].contiguous().view(torch.uint8)), x


# a call's most rows: one workgroup selects among them, or splits do
@pytest.mark.parametrize("max_rows", [256, 9000])
def test_counters_below_zero_pass_through(max_rows):
    """A slot with rows < 0 is one that the other calls skip; adopting rows_out leaves it so."""
    p = params(4, 2, 64, "f32", sink=3, recent=9, topk=40)
    print(f"\n[case] evict, rows -1 and -2147483648, at most {max_rows}", flush=True)
    rows = [-1, 40, -(1 << 31), 0]
    c, state, out, kept = _run(p, "f32", 32, [max_rows, 64, 0, 0], rows, max_rows)
    assert out == [-1, 40, -(1 << 31), 0]
    assert (kept[[0, 2, 3]] == -1).all() and (kept[1] == np.where(np.arange(p.budget) < 40, np.arange(p.budget), -1)).all()
    _same(state, c.state())


@pytest.mark.parametrize("topk,max_rows,rows", [(40, 20, [50, 52, 20, 60]), (9000, 8500, [8900, 9012, 100, 9100])])
def test_max_rows_below_the_budget_drops_no_row(topk, max_rows, rows):
    """Slots within the budget are left alone, though they hold more rows than the call looks at; of one over it the
    first budget rows stay."""
    p = params(4, 2, 64, "f32", sink=3, recent=9, topk=topk)
    B = p.budget
    assert B == topk + 12 and max_rows < B
    print(f"\n[case] evict, rows {rows} of which {max_rows} are looked at, budget {B}", flush=True)
    c, state, out, kept = _run(p, "f32", 32, rows, rows, max_rows)
    assert out == [min(r, B) for r in rows]
    for b, r in enumerate(rows):
        assert (kept[b] == np.where(np.arange(B) < min(r, B), np.arange(B), -1)).all(), b
    _same(state, c.state())


def _expected(token, weight, there, rows, pos, p):
    """kept_out of one (slot, head): rows in pages that are not there are neither kept nor filled."""
    B = p.budget
    if rows <= B:
        return np.array([r if r < rows and there[r] else -1 for r in range(B)])
    r = np.arange(rows)
    safe = there & ((token < p.sink) | (token >= pos - p.recent))
    places = int(there[:B].sum())
    kept = r[safe][:places].tolist()
    others = sorted(r[there & ~safe].tolist(), key=lambda i: (-weight[i], i))
    kept = sorted(kept + others[:max(0, places - int(safe.sum()))])
    out = np.full(B, -1)
    here = [i for i in kept if i < B]
    out[here] = here
    out[np.flatnonzero((out < 0) & there[:B])] = [i for i in kept if i >= B]
    return out


@pytest.mark.parametrize("max_rows", [640, 16384])
@pytest.mark.parametrize("what", ["below", "behind", "protected", "both", "all-below", "all-behind", "all", "ties",
                                  "protected-over-places"])
def test_pages_that_are_not_there(what, max_rows):
    """Pages of 32 rows missing below the budget of 100, behind it, or with the first and latest tokens: no kept row goes
    there, and none comes from there."""
    over = dict(recent=90, topk=7) if what == "protected-over-places" else dict(recent=9, topk=88)
    p = params(4, 2, 64, "bf16", sink=3, **over)
    assert p.budget == 100
    page, rows = 32, [600, 101, 333, 90]
    gone = {"below": [1], "behind": [4, 9], "protected": [0, 18, 10], "both": [2, 3, 5], "all-below": [0, 1, 2, 3],
            "all-behind": list(range(4, 19)), "all": list(range(19)), "ties": [1, 3, 4], "protected-over-places": [0, 2]}[what]
    print(f"\n[case] evict, pages {gone} not there, rows {rows}, at most {max_rows}", flush=True)

    def before(c):
        g = torch.Generator().manual_seed(9)
        w = torch.rand(c.weight.shape, generator=g)
        if what == "ties":
            w = torch.round(w * 2) / 2  # many zeros among them
        c.weight.copy_(w)
        for i, j in enumerate(gone):
            c.table[:, j] = [-1, c.n_pages, -(1 << 31), (1 << 31) - 1][i % 4]

    c, state, out, kept = _run(p, "bf16", page, [max_rows if b == 0 else x for b, x in enumerate(rows)], rows, max_rows,
                               before=before)
    assert out == [min(r, 100) for r in rows]
    want = {x: state[x].clone() for x in ("k", "v", "token", "weight", "rows", "pos")}
    for b, R in enumerate(rows):
        pl = c.places(b, R)
        for h in range(p.n_kv_heads):
            (token, there), weight = c.gather("token", b, h, R, state), c.gather("weight", b, h, R, state)[0]
            exp = _expected(token.numpy(), weight.numpy(), there, R, R + 30, p)
            assert (kept[b, h] == exp).all(), (b, h, np.flatnonzero(kept[b, h] != exp)[:5])
            for to in np.flatnonzero((exp >= 0) & (exp != np.arange(100))):
                for x in ("k", "v", "token", "weight"):
                    want[x][pl[to][0], h, pl[to][1]] = state[x][pl[exp[to]][0], h, pl[exp[to]][1]]
    _same(want, c.state())
