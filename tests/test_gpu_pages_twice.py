"""Slots that a page-table call names more than once, near one another and more than a wave or a chunk of sequences apart,
with pages to spare and too few: reserved as by calls one after the other, released once.  Exact, against lists.  Every case
prints what names it before touching the GPU."""
import pytest
import torch

import paper_2511_03092_amd as snap
from test_gpu_pages import Pool, _i32

pytestmark = pytest.mark.gpu


class Twice(Pool):
    def release(self, rows, slots):
        for s in reversed(slots):  # the last one named gives
            if 0 <= s < len(self.table):
                keep = min(len(self.table[s]), -(-max(0, rows[s]) // self.page))
                self.free += self.table[s][keep:][::-1]
                self.table[s] = self.table[s][:keep]

    def check(self):  # (no list is compared in an assertion: pytest would spend minutes on their differences)
        got = {n: t.cpu().tolist() for n, t in self.t.items()}
        same = {"n": got["n"] == [len(self.free)], "free": got["free"][:len(self.free)] == self.free,
                "held": got["held"] == [len(x) for x in self.table],
                "table": got["table"] == [x + [-1] * (self.max_pages - len(x)) for x in self.table]}
        assert all(same.values()), same
        every = sorted([x for t in self.table for x in t] + self.free) == list(range(self.n_pages))
        assert every, "a page is lost or twice"


@pytest.mark.parametrize("pages", [3, 60, 400, 3000])
@pytest.mark.parametrize("n,n_slots", [(5, 2), (64, 40), (130, 64), (200, 7), (1024, 500), (1500, 600), (2500, 2500)])
def test_reserved_in_order_and_released_once(n, n_slots, pages):
    print(f"\n[case] {n} sequences of {n_slots} slots, {pages} pages", flush=True)
    g = torch.Generator().manual_seed(n + pages)
    r = lambda m, k: torch.randint(0, m, (k,), generator=g).tolist()  # noqa: E731
    pool = Twice(n_slots, pages, 16, 7, 1)
    rows = [0] * n_slots
    for step in range(5):
        slots = r(n_slots, n)
        if step % 2:
            slots[n // 2], slots[n // 3] = -1, n_slots
        lengths = r(16 * 9 if step == 3 else 16 * 3, n)  # (of 7 pages at most)
        short = torch.full((n,), -7, dtype=torch.int32, device="cuda")
        snap.snap_pages_reserve(pool.c, _i32(rows), _i32(slots), _i32(lengths), short)
        torch.cuda.synchronize()
        want = pool.reserve(rows, slots, lengths)
        bad = [(b, x, y) for b, (x, y) in enumerate(zip(short.cpu().tolist(), want)) if x != y]
        assert not bad, bad[:5]
        pool.check()
        rows = [min(16 * len(x), 16 * len(x) - y) if x else 0 for x, y in zip(pool.table, r(40, n_slots))]
        if step == 2 and n_slots > 3:
            rows[3] = -1
        gone = r(n_slots, n)
        snap.snap_pages_release(pool.c, _i32(rows), _i32(gone))
        torch.cuda.synchronize()
        pool.release(rows, gone)
        pool.check()
        rows = [max(0, x) for x in rows]
        free = torch.randperm(n_slots, generator=g)[:n_slots // 2].tolist()  # room for the next step
        for s in free:
            rows[s] = 0
        snap.snap_pages_release(pool.c, _i32(rows), _i32(free))
        pool.release(rows, free)
        torch.cuda.synchronize()
        pool.check()


def test_a_refused_wish_leaves_the_pages_of_the_served_one():
    """The first wish of a slot and others more than a wave behind it, some of them more than the pages that are left."""
    print("\n[case] one slot, wishes a wave apart, too few pages", flush=True)
    for pages, first, later in ((3, 64, 32), (3, 32, 64), (4, 64, 32), (2, 32, 64), (5, 32, 80)):
        pool = Twice(300, pages, 16, 8, 2)
        slots = [7] + list(range(10, 210)) + [7] + list(range(210, 280)) + [7]
        lengths = [first] + [0] * 200 + [later] + [0] * 70 + [later]
        short = torch.zeros(len(slots), dtype=torch.int32, device="cuda")
        snap.snap_pages_reserve(pool.c, _i32([0] * 300), _i32(slots), _i32(lengths), short)
        torch.cuda.synchronize()
        assert short.cpu().tolist() == pool.reserve([0] * 300, slots, lengths)
        pool.check()
        snap.snap_pages_release(pool.c, _i32([0] * 300), _i32(slots))
        torch.cuda.synchronize()
        pool.release([0] * 300, slots)
        pool.check()
        assert int(pool.t["n"]) == pages
