"""The block cache (snap_block_*) against its definition: codes, scales, bounds, tails and selections exactly, attention
in float64 with tolerances by arithmetic (blockhelp).  Every case prints what names it before touching the GPU."""
import pytest
import torch

import paper_2511_03092_amd as snap
from blockhelp import Blocks, check_out, params

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _rand(g, *shape, spread=True):
    x = torch.randn(shape, generator=g)
    if spread:  # some dims larger than others
        x = x * (0.25 + 3 * torch.rand(shape[-1:], generator=g) ** 4)
    return x.bfloat16()


def _load(c, slots, lengths, seed, like=None):
    """Random rows stored in slots by one call; rows advanced."""
    g = torch.Generator().manual_seed(seed)
    h, d = c.p.n_kv_heads, c.p.d_qk
    m = max(1, max(lengths))
    k, v = (_rand(g, len(slots), h, m, d) if like is None else like[i] for i in range(2))
    snap.snap_block_append(c.p, c.c, c.rows, _i32(slots), k.cuda(), v.cuda(), lengths=_i32(lengths))
    for b, (s, n) in enumerate(zip(slots, lengths)):
        if 0 <= s < c.n_slots and n > 0 and int(c.rows[s]) >= 0:
            c.put(s, k[b, :, :n].transpose(0, 1), v[b, :, :n].transpose(0, 1))
            c.rows[s] += n
    return k, v


def _call(c, slots, q, max_rows=None, select=False, new=None, dtype=torch.bfloat16, ws=None):
    """attn, or step with new = (k, v); out and selections."""
    n, p = len(slots), c.p
    mr = max_rows or c.max_pages * c.page
    out = torch.full((n, p.n_q_heads, p.d_qk), float("nan"), dtype=dtype, device="cuda")
    sel = torch.full((n, p.n_kv_heads, snap.snap_block_chosen(p, c.block)), -7, dtype=torch.int32, device="cuda") if select else None
    if ws is None:
        ws = snap.workspace(snap.snap_block_decode_workspace(p, n, mr, c.block, select))
        ws.fill_(255)  # NaN in every float
    if new is None:
        snap.snap_block_decode_attn(p, c.c, c.rows, _i32(slots), q, out, ws, max_rows=mr, select=select, sel_out=sel)
    else:
        snap.snap_block_decode_step(p, c.c, c.rows, _i32(slots), q, *new, out, ws, max_rows=mr, select=select, sel_out=sel)
    torch.cuda.synchronize()
    return out, sel


SHAPES = [("i8", 128, 64, 64), ("i8", 64, 32, 128), ("fp8", 128, 32, 32), ("fp8", 64, 128, 256), ("bf16", 128, 64, 128),
          ("bf16", 64, 32, 64), ("i8", 128, 128, 128)]


# ---------------------------------------------------------------- storing
@pytest.mark.parametrize("kv,d,block,page", SHAPES)
@pytest.mark.parametrize("calls", [[300], [1] * 70, [31, 1, 1, 64, 5, 128, 63], [0, 129, 0, 127], [1, 255]], ids=str)
def test_rows_are_stored_the_same_however_they_are_split(kv, d, block, page, calls):
    print(f"\n[case] block append {kv} d {d} block {block} page {page}, calls of {calls[:8]} tokens", flush=True)
    p = params(4, 2, d, kv)
    c = Blocks(p, kv, block, page, [0, 320, 330], 1)
    before = c.state()
    for i, n in enumerate(calls):
        _load(c, [2, 1], [n, max(0, n - 1)], 10 + i)
        torch.cuda.synchronize()
    c.check(before)


@pytest.mark.parametrize("kv,d,block,page", SHAPES[:5])
def test_packed_and_strided_inputs_store_the_same(kv, d, block, page):
    print(f"\n[case] block append {kv} d {d} block {block}: packed and strided inputs", flush=True)
    p, lengths = params(6, 3, d, kv), [70, 0, 301, 1]
    g = torch.Generator().manual_seed(3)
    rows = [_rand(g, n, 2 * 3, d) for n in lengths]
    packed = torch.cat(rows)
    padded = torch.zeros((4, 6, 320, d), dtype=torch.bfloat16)
    for b, x in enumerate(rows):
        padded[b, :, :len(x)] = x.transpose(0, 1)
    slots = [3, 0, 1, 4]
    starts = _i32([0, 70, 70, 371, 372])
    states = []
    for form in ("packed", "padded", "token-major"):
        c = Blocks(p, kv, block, page, [60, 340, 10, 200, 64], 1)
        before = c.state()
        _load(c, slots, [33, 5, 17, 0], 5)
        if form == "packed":
            x = packed.cuda()
            snap.snap_block_append(p, c.c, c.rows, _i32(slots), x[:, :3], x[:, 3:], starts=starts, max_len=301)
        else:
            x = padded.cuda()
            if form == "token-major":
                x = x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
            snap.snap_block_append(p, c.c, c.rows, _i32(slots), x[:, :3], x[:, 3:], lengths=_i32(lengths))
        torch.cuda.synchronize()
        for s, y in zip(slots, rows):
            c.put(s, y[:, :3], y[:, 3:])
        states.append(c.check(before))
    for st in states[1:]:
        for n in st:
            assert torch.equal(st[n].contiguous().view(torch.uint8), states[0][n].contiguous().view(torch.uint8)), n


@pytest.mark.parametrize("kv", ["i8", "fp8", "bf16"])
def test_slots_pages_and_rows_that_are_not_there(kv):
    """Slot ids out of range, negative counters, holes, rows past the table, starts out of order."""
    print(f"\n[case] block append {kv}: what is not there", flush=True)
    p = params(4, 2, 64, kv)
    c = Blocks(p, kv, 32, 64, [256, 256, 256, 128], 2, holes=[(0, 1), (1, 3), (1, 0)], max_pages=4)
    before = c.state()
    c.rows[2] = -1
    g = torch.Generator().manual_seed(7)
    k, v = _rand(g, 5, 2, 260, 64), _rand(g, 5, 2, 260, 64)
    slots = [0, 2, 9, 1, -1]
    snap.snap_block_append(p, c.c, c.rows, _i32(slots), k.cuda(), v.cuda(), lengths=_i32([200, 100, 50, 300, 10]))
    torch.cuda.synchronize()
    for b, n in ((0, 200), (3, 256)):
        c.put(slots[b], k[b, :, :n].transpose(0, 1), v[b, :, :n].transpose(0, 1))
    c.check(before)
    tails = c.state()
    if kv != "bf16":  # slot 1's last block is in a page that is not there; slots 2 and 3 had no call
        for s in (1, 2, 3):
            assert torch.isnan(tails["k_tail"][s]).all()
    x = k[0].transpose(0, 1).contiguous().cuda()
    snap.snap_block_append(p, c.c, c.rows, _i32([3, 3]), x, x, starts=_i32([50, 20, 900]), max_len=10)  # -30 and 240 tokens
    torch.cuda.synchronize()
    y = x[20:30].cpu()
    c.put(3, y, y)
    c.check(before)


@pytest.mark.parametrize("kv", ["i8", "fp8"])
def test_values_of_every_size(kv):
    """Zero blocks, the least and largest of the type, infinities and NaN."""
    print(f"\n[case] block append {kv}: values of every size", flush=True)
    p = params(2, 1, 64, kv)
    c = Blocks(p, kv, 32, 32, [32 * 12], 4)
    before = c.state()
    g = torch.Generator().manual_seed(8)
    x = _rand(g, 12, 32, 64, spread=False).float()
    x[0] = 0
    x[1] *= 1e-39
    x[2] *= 2.0 ** -126
    x[3] *= 1e37
    x[4] = 0
    x[4, 3, 5] = -3.3e38
    x[5, 1, 2], x[5, 7, 2], x[5, 9, 4] = float("inf"), -float("inf"), float("nan")
    x[6, :, 9] = float("nan")
    x[7] = float("nan")
    x[8] = float("inf")
    x[9] = 1.0
    x[10] = torch.arange(64).float() - 31.5  # quotients that are ties or near them
    x[11] *= 1e-41
    x = x.bfloat16().reshape(1, 1, 12 * 32, 64)
    _load(c, [0], [12 * 32], 1, like=(x, x.flip(2)))
    torch.cuda.synchronize()
    c.check(before)


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("kv,d,block,page", SHAPES)
@pytest.mark.parametrize("hq,hkv", [(4, 2), (16, 1), (3, 3), (10, 2)])
def test_attention_over_every_block(kv, d, block, page, hq, hkv, dtype):
    lengths = [1, 0, 31, 32, 33, 64, 65, 127, 128, 129, 700, 1025, 257]
    print(f"\n[case] block attention {kv} d {d} block {block} page {page} heads {hq}/{hkv}", flush=True)
    p = params(hq, hkv, d, kv)
    c = Blocks(p, kv, block, page, [max(1, n) for n in lengths], 5, bounds=False)
    slots = list(range(len(lengths)))
    _load(c, slots, lengths, 6)
    c.rows -= 1  # the newest token is stored already
    q = (2 * _rand(torch.Generator().manual_seed(9), len(slots), hq, d, spread=False)).cuda()
    out, _ = _call(c, slots, q, dtype=dtype)
    check_out(c, slots, [n - 1 for n in lengths], q, out, c.max_pages * c.page)


@pytest.mark.parametrize("kv", ["i8", "fp8", "bf16"])
def test_attention_with_holes_bounds_and_bad_slots(kv):
    """Pages that are not there, slot ids out of range, a bound below the rows held."""
    print(f"\n[case] block attention {kv}: holes, bad slots, bounds", flush=True)
    p = params(8, 2, 128, kv)
    c = Blocks(p, kv, 64, 128, [600, 600, 640, 130], 6, holes=[(0, 0), (0, 2), (1, 4), (3, 0), (3, 1)])
    lengths = [600, 600, 640, 130]
    _load(c, [0, 1, 2, 3], lengths, 7)
    c.rows -= 1
    slots = [3, 0, -5, 1, 2, 4]
    rows = [129, 599, None, 599, 639, None]
    g = torch.Generator().manual_seed(1)
    q = _rand(g, len(slots), 8, 128).cuda()
    real = [s if 0 <= s < 4 else 0 for s in slots]
    for mr in (640, 600, 513, 130, 64, 1):
        out, _ = _call(c, slots, q, max_rows=mr, dtype=torch.float32)
        check_out(c, real, rows, q, out, mr)


@pytest.mark.parametrize("select", [False, True], ids=["all", "select"])
@pytest.mark.parametrize("kv,d,block,page", SHAPES)
def test_a_step_is_an_append_and_an_attention(kv, d, block, page, select):
    """Bit for bit, over the ends of blocks and pages."""
    print(f"\n[case] block step {kv} d {d} block {block} page {page} select {select}", flush=True)
    p = params(8, 2, d, kv, sink=4, recent=40, topk=2 * block)
    lengths, slots = [block - 2, 5 * block + 1, 0, 2 * page - 2], [2, 0, 3, 1]
    both = [Blocks(p, kv, block, page, [8 * block + 4, 2 * page + 8, block + 8, 8], 7) for _ in range(2)]
    before = both[0].state()
    for c in both:
        _load(c, slots, lengths, 8)
    g = torch.Generator().manual_seed(2)
    for step in range(5):
        q = _rand(g, 4, 8, d).cuda()
        k, v = _rand(g, 4, 2, 1, d), _rand(g, 4, 2, 1, d)
        one, two = both
        snap.snap_block_append(p, one.c, one.rows, _i32(slots), k.cuda(), v.cuda())
        a, sa = _call(one, slots, q, select=select)
        b, sb = _call(two, slots, q, select=select, new=(k.cuda(), v.cuda()))
        assert torch.equal(a.view(torch.int16), b.view(torch.int16)), step
        assert not select or torch.equal(sa, sb)
        rows = one.rows.cpu()
        for c in both:
            for i, s in enumerate(slots):
                c.put(s, k[i, :, :].transpose(0, 1), v[i].transpose(0, 1))
        check_out(one, slots, [int(rows[s]) if int(rows[s]) < one.max_pages * page else None for s in slots], q, a,
                  one.max_pages * page, select, sa)
        for c in both:
            snap.snap_advance(c.rows, _i32(slots))
    x, y = (c.check(before) for c in both)
    for n in x:
        assert torch.equal(x[n].contiguous().view(torch.uint8), y[n].contiguous().view(torch.uint8)), n


# ---------------------------------------------------------------- selection
@pytest.mark.parametrize("sink,recent,topk", [(4, 8, 100), (0, 1, 0), (0, 1, 1), (100, 100, 320), (1000, 1, 64), (0, 5000, 64),
                                              (4, 300, 5000), (64, 64, 64)])
@pytest.mark.parametrize("kv,d,block,page,hq", [("i8", 128, 32, 64, 8), ("fp8", 64, 64, 64, 6), ("bf16", 128, 64, 128, 32),
                                                ("i8", 64, 128, 128, 2)])
def test_selected_blocks(kv, d, block, page, hq, sink, recent, topk):
    print(f"\n[case] block select {kv} d {d} block {block} sink {sink} recent {recent} topk {topk}", flush=True)
    p = params(hq, 2, d, kv, sink=sink, recent=recent, topk=topk)
    lengths = [2000, 1, block, block + 1, 0, 1999, 900]
    c = Blocks(p, kv, block, page, [max(1, n) for n in lengths], 8, holes=[(5, 0), (5, 3)])
    slots = list(range(len(lengths)))
    _load(c, slots, lengths, 9)
    c.rows -= 1
    q = _rand(torch.Generator().manual_seed(3), len(slots), hq, d).cuda()
    out, sel = _call(c, slots, q, select=True, dtype=torch.float32)
    check_out(c, slots, [n - 1 for n in lengths], q, out, c.max_pages * c.page, True, sel)


@pytest.mark.parametrize("what", ["equal", "two", "zero-q", "nan-q", "tiny", "negative"])
def test_selection_of_equal_and_odd_scores(what):
    """Ties go to the lower block, whatever the scores' sign and size."""
    print(f"\n[case] block select: {what}", flush=True)
    p = params(4, 2, 64, "i8", sink=0, recent=1, topk=7 * 32)
    c = Blocks(p, "i8", 32, 32, [32 * 60 + 5], 9)
    g = torch.Generator().manual_seed(4)
    n = 32 * 60 + 5
    k = _rand(g, 1, 2, n, 64)
    if what == "equal":
        k = k[:, :, :32].repeat(1, 1, 61, 1)[:, :, :n].contiguous()
    elif what == "two":
        k = torch.cat((k[:, :, :32], k[:, :, 32:64]), 2).repeat(1, 1, 31, 1)[:, :, :n].contiguous()
    elif what == "tiny":
        k = (k.float() * 1e-30).bfloat16()
    elif what == "negative":
        k = (-k.float().abs() - 1).bfloat16()
    _load(c, [0], [n], 1, like=(k, _rand(g, 1, 2, n, 64)))
    c.rows -= 1
    q = _rand(g, 1, 4, 64)
    if what == "zero-q":
        q.zero_()
    elif what == "nan-q":
        q[0, 0, 3], q[0, 1, 5], q[0, 2, 0] = float("nan"), float("inf"), -float("inf")
    elif what == "tiny":
        q = (q.float() * 1e-30).bfloat16()
    elif what == "negative":
        q = q.abs()
    out, sel = _call(c, [0], q.cuda(), select=True, dtype=torch.float32)
    if what == "nan-q":
        from blockhelp import choose
        for h in range(2):
            assert sel[0, h].cpu().tolist()[:7] == choose(c, 0, h, n - 1, q[0, 2 * h:2 * h + 2], n)
    else:
        check_out(c, [0], [n - 1], q.cuda(), out, c.max_pages * c.page, True, sel)


@pytest.mark.parametrize("kv", ["i8", "bf16"])
def test_counters_far_past_the_cache(kv):
    """A slot whose counter is the largest number, beside a sound one: its whole blocks below the bound, nothing stored."""
    print(f"\n[case] block step {kv}: counters past the cache", flush=True)
    p = params(4, 2, 64, kv, sink=40, recent=1 << 23, topk=100)
    c = Blocks(p, kv, 32, 64, [256, 256], 9, max_pages=4)
    before = c.state()
    _load(c, [0, 1], [256, 100], 2)
    c.rows[0] = 2 ** 31 - 1
    g = torch.Generator().manual_seed(5)
    q, new = _rand(g, 2, 4, 64).cuda(), [_rand(g, 2, 2, 1, 64).cuda() for _ in range(2)]
    for n in (0, 1):
        c.put(1, *(x[1].cpu().transpose(0, 1) for x in new)) if n else None
        for select, recent in ((False, 1), (True, 1 << 23), (True, 5)):
            p.recent = recent
            out, sel = _call(c, [0, 1], q, select=select, new=new if not n else None, dtype=torch.float32)
            if n:
                check_out(c, [0, 1], [2 ** 31 - 1, 100], q, out, 256, select, sel)
    c.check(before)


def test_selection_among_the_most_blocks():
    """32768 blocks of one sequence; more are refused."""
    print("\n[case] block select among 32768 blocks", flush=True)
    n = 32768 * 32
    p = params(2, 1, 64, "i8", sink=0, recent=1, topk=64 * 32)
    c = Blocks(p, "i8", 32, 4096, [n + 4096], 10)
    g = torch.Generator().manual_seed(5)
    x = _rand(g, 1, 1, 32 * 4096, 64)
    for _ in range(8):
        _load(c, [0], [32 * 4096], 1, like=(x, x))
    c.x = {m: [y[0]] for m, y in c.x.items()}
    q = _rand(g, 1, 2, 64).cuda()
    c.rows.fill_(n)
    _load(c, [0], [1], 1, like=(x[:, :, :1], x[:, :, :1]))
    c.rows.fill_(n - 1)  # 32767 whole blocks before the newest row's
    out, sel = _call(c, [0], q, max_rows=n, select=True, dtype=torch.float32)
    # every block stands there eight times: the best eight eighths, lower ones first
    from blockhelp import scores
    s = scores(c, 0, 0, q[0].cpu(), range(4096))
    best = sorted(range(4096), key=lambda i: (-float(s[i]), i))
    want = []
    for i in best:
        want += [i + 4096 * r for r in range(8) if i + 4096 * r < 32767]
    have = [j for j in sel[0, 0].cpu().tolist() if j >= 0]
    assert have == sorted(sorted(want[:64]))
    with pytest.raises(snap.SnapError) as e:
        _call(c, [0], q, max_rows=n + 32, select=True)
    assert e.value.status == snap.SNAP_ERR_UNSUPPORTED


def test_pages_past_4_gb():
    """Codes, scales and bounds whose offsets pass 32 bits."""
    print("\n[case] block cache of more than 4 GB a tensor", flush=True)
    p = params(8, 2, 128, "i8", sink=0, recent=1, topk=128)
    c = Blocks(p, "i8", 64, 4096, [9000], 11, n_pages=4500)
    assert c.k.numel() > 1 << 32 and int(c.table_cpu[0, :3].min()) > 4400
    _load(c, [0], [9000], 12)
    c.rows -= 1
    q = _rand(torch.Generator().manual_seed(6), 1, 8, 128).cuda()
    for select in (False, True):
        out, sel = _call(c, [0], q, select=select, dtype=torch.float32)
        check_out(c, [0], [8999], q, out, c.max_pages * c.page, select, sel)
