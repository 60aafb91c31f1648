"""Page tables on the device (snap_pages_*) and the packed append that reads their map, against plain Python.  Every case
prints what names it before touching the GPU."""
import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import IN, Paged, params

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Pool:
    """A pool on the device and the same in Python lists."""

    def __init__(self, n_slots, n_pages, page, max_pages, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.page, self.max_pages, self.n_pages = page, max_pages, n_pages
        self.free = torch.randperm(n_pages, generator=g).tolist()
        self.table = [[] for _ in range(n_slots)]
        self.t = dict(table=torch.full((n_slots, max_pages), -1, dtype=torch.int32, device="cuda"),
                      held=torch.zeros(n_slots, dtype=torch.int32, device="cuda"), free=_i32(self.free), n=_i32([n_pages]))
        self.c = snap.page_pool_struct(self.t["table"], self.t["held"], self.t["free"], self.t["n"], page)

    def reserve(self, rows, slots, lengths):
        short, lacked, free = [], 0, len(self.free)
        for s, n in zip(slots, lengths):
            if not 0 <= s < len(self.table) or rows[s] < 0:
                short.append(0)
                continue
            want = -(-(rows[s] + max(0, n)) // self.page)
            lack = max(0, want - len(self.table[s]))
            if want > self.max_pages:
                short.append(lack)
                continue
            lacked += lack
            if lack and lacked > free:
                short.append(lack)
                continue
            self.table[s] += [self.free.pop() for _ in range(lack)]
            short.append(0)
        return short

    def release(self, rows, slots):
        back = []
        for s in slots:
            if 0 <= s < len(self.table):
                keep = min(len(self.table[s]), -(-max(0, rows[s]) // self.page))
                back += self.table[s][keep:]
                self.table[s] = self.table[s][:keep]
        self.free += back[::-1]

    def check(self):
        assert int(self.t["n"]) == len(self.free)
        assert self.t["free"][:len(self.free)].cpu().tolist() == self.free
        assert self.t["held"].cpu().tolist() == [len(x) for x in self.table]
        assert self.t["table"].cpu().tolist() == [x + [-1] * (self.max_pages - len(x)) for x in self.table]


def _map(pool, rows, pos, slots, lengths, tokens):
    starts, seq, row, at = [0], [], [], []
    for b, (s, n) in enumerate(zip(slots, lengths)):
        ok = 0 <= s < len(pool.table) and rows[s] >= 0
        for t in range(max(0, n)):
            r = rows[s] + t if ok else 0
            j = r // pool.page
            seq.append(b)
            row.append(pool.table[s][j] * pool.page + r % pool.page if ok and j < len(pool.table[s]) else -1)
            at.append((rows[s] if pos is None else pos[s]) + t if ok else 0)
        starts.append(len(seq))
    more = max(0, tokens - len(seq))
    return ([min(x, tokens) for x in starts], (seq + [-1] * more)[:tokens], (row + [-1] * more)[:tokens],
            (at + [0] * more)[:tokens])


def _check_map(pool, rows, pos, slots, lengths, tokens):
    n = len(slots)
    got = [torch.full((m,), -9, dtype=torch.int32, device="cuda") for m in (n + 1, tokens, tokens, tokens)]
    snap.snap_pages_map(pool.c, _i32(rows), _i32(slots), _i32(lengths), *got, pos=None if pos is None else _i32(pos))
    torch.cuda.synchronize()
    for name, x, y in zip(("starts", "seq_of", "row_of", "pos_of"), got, _map(pool, rows, pos, slots, lengths, tokens)):
        assert x.cpu().tolist() == y, name


@pytest.mark.parametrize("page,n_slots,seed", [(16, 5, 0), (64, 70, 1), (4096, 3, 2), (16, 1500, 3), (32, 1025, 4)])
def test_pages_are_handed_out_and_taken_back(page, n_slots, seed):
    """Random growth and release against the lists, with too few pages at times."""
    print(f"\n[case] pages of {page} rows, {n_slots} slots", flush=True)
    g = torch.Generator().manual_seed(seed)
    r = lambda m, k: torch.randint(0, m, (k,), generator=g).tolist()  # noqa: E731
    pool = Pool(n_slots, 3 * n_slots + 7, page, 6, seed)
    rows = [0] * n_slots
    for step in range(8):
        n = max(1, r(n_slots + 1, 1)[0])
        slots = torch.randperm(n_slots, generator=g)[:n].tolist()
        if step % 3 == 1:
            slots[0], slots[-1] = (-1, n_slots)[step % 2], 2 ** 31 - 1
        lengths = r(3 * page, n)
        if step == 4:
            lengths = [1] * n
        short = torch.full((n,), -7, dtype=torch.int32, device="cuda")
        snap.snap_pages_reserve(pool.c, _i32(rows), _i32(slots), 1 if step == 4 else _i32(lengths), short)
        torch.cuda.synchronize()
        want = pool.reserve(rows, slots, lengths)
        assert short.cpu().tolist() == want
        pool.check()
        _check_map(pool, rows, [x + 5 for x in rows] if step % 2 else None, slots, lengths, sum(lengths) + 3)
        for s, x, y in zip(slots, lengths, want):
            if 0 <= s < n_slots and not y:
                rows[s] += x
        if step % 2:
            gone = torch.randperm(n_slots, generator=g)[:max(1, n // 2)].tolist() + [-3]
            for s in gone[:-1]:
                rows[s] = 0 if s % 2 else rows[s] // 2
            snap.snap_pages_release(pool.c, _i32(rows), _i32(gone))
            torch.cuda.synchronize()
            pool.release(rows, gone)
            pool.check()


def test_release_undoes_reserve():
    print("\n[case] pages reserved and released again", flush=True)
    pool = Pool(2100, 9000, 64, 8)
    first = {k: v.clone() for k, v in pool.t.items()}
    slots, rows = torch.randperm(2100).tolist(), _i32([0] * 2100)
    snap.snap_pages_reserve(pool.c, rows, _i32(slots), _i32([(7 * b) % 250 for b in range(2100)]))
    assert int(pool.t["n"]) < 9000
    snap.snap_pages_release(pool.c, rows, _i32(slots))
    torch.cuda.synchronize()
    for k, v in first.items():
        assert torch.equal(pool.t[k], v), k


def test_requests_that_cannot_be_served():
    """A table that is too short, a negative counter and length, lengths that overflow, no free page at all."""
    print("\n[case] pages: requests that cannot be served", flush=True)
    pool = Pool(6, 8, 16, 4)
    rows = [0, 0, -1, 60, 2 ** 31 - 1, 5]
    slots, lengths = [0, 1, 2, 3, 4, 5], [65, 33, 10, 4, 2 ** 31 - 1, -4]
    short = torch.zeros(6, dtype=torch.int32, device="cuda")
    snap.snap_pages_reserve(pool.c, _i32(rows), _i32(slots), _i32(lengths), short)
    torch.cuda.synchronize()
    assert short.cpu().tolist() == pool.reserve(rows, slots, lengths) == [5, 0, 0, 0, 2 ** 28, 0]
    pool.check()
    snap.snap_pages_reserve(pool.c, _i32([0] * 6), _i32([0, 5, 1]), _i32([16, 0, 48]), short[:3])
    torch.cuda.synchronize()
    assert short[:3].cpu().tolist() == pool.reserve([0] * 6, [0, 5, 1], [16, 0, 48]) == [1, 0, 0]
    pool.check()


def test_a_slot_named_twice():
    """Its pages are handed out and taken back once."""
    print("\n[case] pages: a slot named twice", flush=True)
    pool = Pool(5, 20, 16, 8)
    slots = [1, 3, 1, 4, 3]
    snap.snap_pages_reserve(pool.c, _i32([0] * 5), _i32(slots), _i32([50, 30, 20, 10, 64]))
    torch.cuda.synchronize()
    held, table = pool.t["held"].cpu().tolist(), pool.t["table"].cpu()
    assert held == [0, 4, 0, 4, 1] and int(pool.t["n"]) == 20 - 9
    used = [int(table[s, j]) for s in (1, 3, 4) for j in range(held[s])]
    left = pool.t["free"][:11].cpu().tolist()
    assert sorted(used + left) == list(range(20)) and int((table >= 0).sum()) == 9
    snap.snap_pages_release(pool.c, _i32([0, 17, 0, 0, 16]), _i32([1, 3, 3, 1, 1]))
    torch.cuda.synchronize()
    assert pool.t["held"].cpu().tolist() == [0, 2, 0, 0, 1] and int(pool.t["n"]) == 17
    table = pool.t["table"].cpu()
    assert sorted(pool.t["free"][:17].cpu().tolist() + table[table >= 0].tolist()) == list(range(20))


@pytest.mark.parametrize("n,tokens", [(1, 1), (1, 0), (3, 5), (300, 5000), (2, 4096), (600, 1), (5, 100000)])
def test_maps(n, tokens):
    print(f"\n[case] map of {n} sequences, room for {tokens} tokens", flush=True)
    g = torch.Generator().manual_seed(n)
    pool = Pool(n + 1, 20 * n, 16, 40, 1)
    slots = torch.randperm(n + 1, generator=g)[:n].tolist()
    rows = torch.randint(0, 60, (n + 1,), generator=g).tolist()
    lengths = torch.randint(-3, 2 * tokens // n + 2, (n,), generator=g).tolist()
    snap.snap_pages_reserve(pool.c, _i32(rows), _i32(slots), 40)
    torch.cuda.synchronize()
    pool.reserve(rows, slots, [40] * n)
    _check_map(pool, rows, None, slots, lengths, tokens)
    if n > 2:
        rows[slots[1]] = -5
        _check_map(pool, rows, [3 * x for x in range(n + 1)], slots[:-1] + [-1], lengths, tokens)
        _check_map(pool, rows, None, [], [], tokens)


SHAPES = {"bf16": (4, 128, False), "fp8": (2, 64, False), "f32": (2, 64, False), "latent": (1, 576, True), "latent8": (1, 576, True)}


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("split", [False, True], ids=["whole", "views"])
def test_a_packed_batch_is_stored_by_its_map(name, split):
    """The same bytes as the padded append; tokens without a row, sequence or slot are left out."""
    h, d, latent = SHAPES[name]
    kv = {"latent": "bf16", "latent8": "fp8"}.get(name, name)
    print(f"\n[case] packed append {name} {'views' if split else 'whole'}", flush=True)
    p = params(h, h, d, kv, latent)
    lengths, slots, held = [70, 1, 0, 33], [2, 0, 3, 1], [5, 16, 0, 31]
    g = torch.Generator().manual_seed(2)
    total, dv = sum(lengths), 0 if latent else d
    x = torch.randn((total, h * (d + dv)), generator=g).to(IN[kv]).cuda()
    k, v = x[:, :h * d].unflatten(-1, (h, d)), None if latent else x[:, h * d:].unflatten(-1, (h, d))
    if not split:
        k, v = k.contiguous(), None if latent else v.contiguous()
    caches = [Paged(p, kv, 5, 32, [40, 70, 80, 10, 0], 3) for _ in range(2)]
    for c in caches:
        for s, r in zip(slots, held):
            c.rows[s], c.pos[s] = r, r + 9
    one, two = caches
    pool = snap.page_pool_struct(two.table, page_size=32)
    maps = [torch.zeros(m, dtype=torch.int32, device="cuda") for m in (5, total + 4, total + 4, total + 4)]
    snap.snap_pages_map(pool, two.rows, _i32(slots), _i32(lengths), *maps, pos=two.pos)
    snap.snap_paged_append_mapped(p, two.c, _i32(slots), *maps[1:], k, v)
    m = max(lengths)
    kp = torch.zeros((4, h, m, d), dtype=k.dtype, device="cuda")
    vp = None if latent else torch.zeros((4, h, m, d), dtype=k.dtype, device="cuda")
    at = 0
    for b, n in enumerate(lengths):
        kp[b, :, :n] = k[at:at + n].transpose(0, 1)
        if not latent:
            vp[b, :, :n] = v[at:at + n].transpose(0, 1)
        at += n
    snap.snap_paged_append(p, one.c, one.rows, one.pos, _i32(slots), kp, vp, lengths=_i32(lengths))
    torch.cuda.synchronize()
    a, b = one.state(), two.state()
    for y in ("k", "v", "token", "weight"):
        assert a[y] is None or torch.equal(a[y].contiguous().view(torch.uint8), b[y].contiguous().view(torch.uint8)), y
    # rows, sequences and slots out of range store nothing
    seq = torch.where(torch.arange(total, device="cuda") % 3 == 0, 4, -1).to(torch.int32)
    snap.snap_paged_append_mapped(p, two.c, _i32(slots), seq, maps[2], maps[3], k, v)
    snap.snap_paged_append_mapped(p, two.c, _i32([-1, 9, 5, 2 ** 31 - 1]), *maps[1:], k, v)
    bad = torch.where(torch.arange(total, device="cuda") % 2 == 0, two.n_pages * 32, -1).to(torch.int32)
    snap.snap_paged_append_mapped(p, two.c, _i32(slots), maps[1], bad, maps[3], k, v)
    torch.cuda.synchronize()
    c = two.state()
    for y in ("k", "v", "token", "weight"):
        assert b[y] is None or torch.equal(b[y].contiguous().view(torch.uint8), c[y].contiguous().view(torch.uint8)), y
