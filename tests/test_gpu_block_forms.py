"""The forms that block calls take by their sizes (one launch or two, scored apart or not, many sequences), calls that are
captured, replayed, concurrent or given a stream, and the page tables, appends and attention together.  Every case prints
what names it before touching the GPU."""
import pytest
import torch

import paper_2511_03092_amd as snap
from blockhelp import Blocks, check_out, params
from test_gpu_blocks import _call, _i32, _load, _rand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("select", [False, True], ids=["all", "select"])
@pytest.mark.parametrize("kv,d,block,page", [("i8", 128, 32, 64), ("fp8", 64, 64, 64), ("bf16", 128, 32, 32), ("i8", 64, 128, 256),
                                             ("bf16", 64, 32, 64), ("fp8", 128, 64, 128)])
def test_short_calls_in_one_launch(kv, d, block, page, select):
    """Steps of few units: every end of a block, holes, slots that are not there, no rows."""
    print(f"\n[case] one launch: {kv} d {d} block {block} page {page} select {select}", flush=True)
    p = params(8, 2, d, kv, sink=4, recent=20, topk=64)
    lengths = [0, 1, 31, 32, 63, 64, 100, 127, 128, 150, 200, 200]
    top = 255 if d == 128 else 400
    c = Blocks(p, kv, block, page, [n + 2 for n in lengths], 1, holes=[(11, 0)])
    before = c.state()
    slots = list(range(len(lengths)))
    _load(c, slots, lengths, 2)
    g = torch.Generator().manual_seed(3)
    ids = slots + [-1, len(slots)]
    for step in range(2):
        q = _rand(g, len(ids), 8, d).cuda()
        k, v = _rand(g, len(ids), 2, 1, d), _rand(g, len(ids), 2, 1, d)
        out, sel = _call(c, ids, q, max_rows=min(top, c.max_pages * page), select=select, new=(k.cuda(), v.cuda()),
                         dtype=torch.float32 if step else torch.bfloat16)
        for s in slots:
            c.put(s, k[s].transpose(0, 1), v[s].transpose(0, 1))
        check_out(c, slots + [0, 0], [n + step for n in lengths] + [None, None], q, out, top, select, sel)
        snap.snap_advance(c.rows, _i32(slots))
    c.check(before)


@pytest.mark.parametrize("kv,d,block", [("i8", 128, 64), ("fp8", 64, 32), ("bf16", 64, 128)])
@pytest.mark.parametrize("n,longest", [(140, 1900), (140, 2300), (140, 4500), (66, 900), (66, 2600)])
def test_many_sequences(kv, d, block, n, longest):
    """More sequences than a wave has lanes, of unequal length, one launch and two; a sample against the definition and
    every one against the attention of a call of its own."""
    print(f"\n[case] {n} sequences of up to {longest} rows, {kv} d {d} block {block}", flush=True)
    p = params(4, 2, d, kv)
    lengths = [max(1, (longest * (b * 37 % n)) // n) if b % 9 else 3 for b in range(n)]
    lengths[5] = longest
    c = Blocks(p, kv, block, 128, lengths, 2, bounds=False)
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(1)).tolist()
    _load(c, list(range(n)), lengths, 3)
    c.rows -= 1
    q = _rand(torch.Generator().manual_seed(4), n, 4, d).cuda()
    out, _ = _call(c, slots, q, max_rows=longest, dtype=torch.float32)
    at = [lengths[s] - 1 for s in slots]
    check_out(c, slots, at, q, out, longest, only=set(range(0, n, 11)) | {slots.index(5)})
    few, _ = _call(c, slots[60:70], q[60:70].contiguous(), max_rows=longest, dtype=torch.float32)
    assert (few - out[60:70]).abs().max() <= 2.0 ** -14 * out.abs().max()


@pytest.mark.parametrize("kv,d,block,hq", [("i8", 128, 32, 32), ("bf16", 64, 32, 4)])
def test_selection_scored_apart(kv, d, block, hq):
    """So many blocks that they are scored by a launch of their own; holes, a short and an empty sequence beside."""
    print(f"\n[case] select, scored apart: {kv} d {d} block {block}", flush=True)
    rows = 66000 if d == 128 else 132000  # 512 KB of bounds a unit
    p = params(hq, 2, d, kv, sink=70, recent=300, topk=1000)
    c = Blocks(p, kv, block, 256, [rows, 1, 700, rows - 5], 4, holes=[(0, 3), (0, 60), (3, 0)])
    _load(c, [0, 1, 2, 3], [rows, 0, 700, rows - 5], 5)
    c.rows -= 1
    q = _rand(torch.Generator().manual_seed(6), 4, hq, d).cuda()
    out, sel = _call(c, [3, 1, 2, 0], q, max_rows=rows, select=True, dtype=torch.float32)
    check_out(c, [3, 1, 2, 0], [rows - 6, -1, 699, rows - 1], q, out, rows, True, sel)


def test_selections_of_many_short_sequences_in_a_long_table():
    """Keys of 4096 blocks beside the scoring, few of them there; lists as long as the longest selection."""
    print("\n[case] select, 80 units, a bound of 131072 rows", flush=True)
    p = params(4, 2, 64, "i8", sink=4, recent=64, topk=640)
    lengths = [5000, 0, 1] + [40 * b for b in range(3, 40)]
    c = Blocks(p, "i8", 32, 64, [max(1, n) for n in lengths], 5, max_pages=2048)
    _load(c, list(range(40)), lengths, 6)
    c.rows -= 1
    q = _rand(torch.Generator().manual_seed(7), 40, 4, 64).cuda()
    out, sel = _call(c, list(range(40)), q, max_rows=131072, select=True)
    check_out(c, list(range(40)), [n - 1 for n in lengths], q, out, 131072, True, sel)


@pytest.mark.parametrize("kv", ["i8", "bf16"])
def test_a_packed_batch_of_many_short_sequences_and_a_long_one(kv):
    """No bound on the lengths."""
    print(f"\n[case] packed append {kv}: 70 sequences, one long", flush=True)
    p = params(2, 2, 64, kv)
    lengths = [(7 * b) % 50 for b in range(70)]
    lengths[33] = 4001
    held = [(11 * b) % 40 for b in range(70)]
    c = Blocks(p, kv, 32, 64, [n + m + 1 for n, m in zip(lengths, held)], 5)
    before = c.state()
    _load(c, list(range(70)), held, 6)
    g = torch.Generator().manual_seed(8)
    x = _rand(g, sum(lengths), 4, 64)
    starts = [0]
    for n in lengths:
        starts.append(starts[-1] + n)
    slots = torch.randperm(70, generator=g).tolist()
    dev = x.cuda()
    order = torch.cat([torch.arange(starts[s], starts[s + 1]) for s in slots])
    at = [0]
    for s in slots:
        at.append(at[-1] + lengths[s])
    y = dev[order.cuda()]
    snap.snap_block_append(p, c.c, c.rows, _i32(slots), y[:, :2], y[:, 2:], starts=_i32(at))
    torch.cuda.synchronize()
    for s in range(70):
        c.put(s, x[starts[s]:starts[s + 1], :2], x[starts[s]:starts[s + 1], 2:])
    c.check(before)


def test_slots_that_share_whole_pages():
    """Two slots whose first pages are one slot's: both attend them, and grow into pages of their own."""
    print("\n[case] block cache: shared pages", flush=True)
    p = params(4, 2, 64, "i8", sink=4, recent=8, topk=64)
    c = Blocks(p, "i8", 32, 64, [128, 64, 0], 7, max_pages=4)
    before = c.state()
    k, v = _load(c, [0], [128], 8)
    t = c.table_cpu
    t[1, 2], t[1, :2] = t[1, 0].clone(), t[0, :2]
    c.table.copy_(t)
    c.rows[1] = 128
    c.put(1, k[0].transpose(0, 1), v[0].transpose(0, 1))
    _load(c, [1], [50], 9)
    g = torch.Generator().manual_seed(1)
    c.rows[:2] -= 1
    q = _rand(g, 2, 4, 64).cuda()
    for select in (False, True):
        out, sel = _call(c, [0, 1], q, select=select, dtype=torch.float32)
        check_out(c, [0, 1], [127, 177], q, out, 256, select, sel)
    c.check(before)


@pytest.mark.parametrize("factor", [1e-6, 1e6, 3e37])
def test_scales_of_every_size_and_a_given_softmax_scale(factor):
    """Keys and values far from 1, queries and sm_scale that bring the logits back."""
    print(f"\n[case] block attention: values times {factor}", flush=True)
    p = params(4, 2, 64, "i8", sm_scale=0.05)
    c = Blocks(p, "i8", 32, 32, [400], 8)
    g = torch.Generator().manual_seed(2)
    k, v = (_rand(g, 1, 2, 400, 64).float() for _ in range(2))
    like = ((k * min(factor, 1e6)).bfloat16(), (v * factor * (0.1 + 0.9 * torch.rand(1, 1, 400, 1, generator=g))).bfloat16())
    _load(c, [0], [400], 1, like=like)
    c.rows -= 1
    q = (_rand(g, 1, 4, 64).float() / min(factor, 1e6)).bfloat16().cuda()
    out, _ = _call(c, [0], q, dtype=torch.float32)
    check_out(c, [0], [399], q, out, 416)


def test_a_call_takes_a_stream_and_calls_overlap():
    """Two layers' steps at once on their own streams, with workspaces of their own, give what they give in turn."""
    print("\n[case] block steps on two streams at once", flush=True)
    p = params(8, 2, 128, "i8", sink=4, recent=64, topk=256)
    caches = [Blocks(p, "i8", 64, 64, [3000, 2000, 700], 9 + i) for i in range(2)]
    for i, c in enumerate(caches):
        _load(c, [0, 1, 2], [2900, 1900, 640], 10 + i)
    g = torch.Generator().manual_seed(3)
    q = [_rand(g, 3, 8, 128).cuda() for _ in range(2)]
    new = [tuple(_rand(g, 3, 2, 1, 128).cuda() for _ in range(2)) for _ in range(2)]
    ids, want = _i32([0, 1, 2]), []
    for select in (False, True):
        for i, c in enumerate(caches):
            want.append(_call(c, [0, 1, 2], q[i], select=select, new=new[i])[0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    nbytes = snap.snap_block_decode_workspace(p, 3, 3008, 64, True)
    ws = [snap.workspace(nbytes) for _ in range(2)]
    outs = [torch.zeros_like(x) for x in want]
    torch.cuda.synchronize()
    for _ in range(10):
        for j, select in enumerate((False, True)):
            for i, c in enumerate(caches):
                snap.snap_block_decode_step(p, c.c, c.rows, ids, q[i], *new[i], outs[2 * j + i], ws[i], max_rows=3008, select=select,
                                            stream=streams[i].cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("kv,select", [("i8", True), ("fp8", False), ("bf16", True)])
def test_pages_prompts_and_steps_together(kv, select):
    """A serving loop: room reserved, packed prompts stored by their starts, steps captured into one graph with the pages
    they grow into and replayed, sequences that end and hand their pages to others; every step against the definition."""
    print(f"\n[case] serving loop {kv} select {select}", flush=True)
    p = params(8, 2, 64, kv, sink=4, recent=40, topk=96)
    n_slots, page, block, max_pages = 5, 64, 32, 8
    c = Blocks(p, kv, block, page, [0] * n_slots, 1, n_pages=30, max_pages=max_pages)
    held, free, n_free = (torch.zeros(n_slots, dtype=torch.int32, device="cuda"),
                          torch.randperm(30, generator=torch.Generator().manual_seed(2)).to(torch.int32).cuda(), _i32([30]))
    pool = snap.page_pool_struct(c.table, held, free, n_free, page)
    g = torch.Generator().manual_seed(3)
    ws = snap.workspace(snap.snap_block_decode_workspace(p, 3, max_pages * page, block, select))

    def prompts(slots, lengths):
        total = sum(lengths)
        short = torch.full((len(slots),), -1, dtype=torch.int32, device="cuda")
        maps = [torch.zeros(m, dtype=torch.int32, device="cuda") for m in (len(slots) + 1, total, total, total)]
        snap.snap_pages_reserve(pool, c.rows, _i32(slots), _i32(lengths), short)
        snap.snap_pages_map(pool, c.rows, _i32(slots), _i32(lengths), *maps)
        both = _rand(g, total, 4, 64)
        dev = both.cuda()
        snap.snap_block_append(p, c.c, c.rows, _i32(slots), dev[:, :2], dev[:, 2:], starts=maps[0])
        torch.cuda.synchronize()
        assert short.tolist() == [0] * len(slots)
        c.table_cpu = c.table.cpu()
        seq, row = maps[1].cpu(), maps[2].cpu()
        for b, s in enumerate(slots):
            mine = both[seq == b]
            assert len(mine) == lengths[b]
            r0 = len(c.x["k"][s])
            assert row[seq == b].tolist() == [int(c.table_cpu[s, r // page]) * page + r % page for r in range(r0, r0 + lengths[b])]
            c.put(s, mine[:, :2], mine[:, 2:])
            c.rows[s] += lengths[b]

    slots = [4, 0, 2]
    ids = _i32(slots)
    prompts(slots, [200, 61, 1])
    q, k, v = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((3, 8, 64), (3, 2, 1, 64), (3, 2, 1, 64)))
    out = torch.zeros((3, 8, 64), dtype=torch.bfloat16, device="cuda")
    sel = torch.zeros((3, 2, snap.snap_block_chosen(p, block)), dtype=torch.int32, device="cuda") if select else None

    def step():
        snap.snap_pages_reserve(pool, c.rows, ids, 1)
        snap.snap_block_decode_step(p, c.c, c.rows, ids, q, k, v, out, ws, select=select, sel_out=sel)
        snap.snap_advance(c.rows, ids)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        step()
    for i in range(70):
        rows = c.rows.cpu().tolist()
        for x in (q, k, v):
            x.copy_(_rand(g, *x.shape))
        graph.replay() if i % 3 else step()
        torch.cuda.synchronize()
        c.table_cpu = c.table.cpu()
        for b, s in enumerate(slots):
            c.put(s, k[b].transpose(0, 1), v[b].transpose(0, 1))
        if i % 7 == 0 or i > 60:
            check_out(c, slots, [rows[s] for s in slots], q, out, max_pages * page, select, sel)
        if i == 40:  # slot 4 ends; its pages go to a new prompt of slot 4 and one of slot 1
            snap.snap_pages_release(pool, torch.where(torch.arange(n_slots, device="cuda") == 4, 0, c.rows).to(torch.int32), _i32([4]))
            c.rows[4] = 0
            for n in ("k", "v"):
                c.x[n][4] = c.x[n][4][:0]
            prompts([1, 4], [100, 33])
    assert int(n_free) == 30 - int(held.sum())
    used = c.table.cpu()[c.table.cpu() >= 0].tolist()
    assert len(set(used)) == len(used)


def test_the_debug_build_records_nothing():
    """The cut's and the selection's invariants, on the build that checks them."""
    print("\n[case] block calls on the debug build", flush=True)
    prev = snap.use_library(snap.DEBUG_LIB_PATH)
    try:
        snap.snap_debug_checks()
        test_many_sequences("i8", 128, 64, 66, 2600)
        test_selection_scored_apart("bf16", 64, 32, 4)
        test_short_calls_in_one_launch("fp8", 64, 64, 64, True)
        assert snap.snap_debug_checks() == 0
    finally:
        snap._lib = prev
