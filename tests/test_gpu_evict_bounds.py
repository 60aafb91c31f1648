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
