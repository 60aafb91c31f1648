"""What attention over the block cache computes with 32 bits: values of every size, in 8 bits and as they came, keep the
errors of fp32 sums; probabilities enter the value product whole; infinities and NaN show where the definition has them.
Every case prints what names it before touching the GPU.

Tolerances, by arithmetic (u = 2^-24, a rounding to fp32 is off by at most u relative), for n rows:
  * a logit z = scale q.k of d products added in fp32 is off by at most dz = scale (d + 4) u sum|q_i k_i|, a probability by
    2 dz + 64 u (the exponent's rounding, for |z| below 64) + 16 u (exp2, references, scales, reciprocals, products),
  * the two sums by u for each addition on a term's way (32-row steps, the 37 of lanes, waves or items), each:
    2 (n / 32 + 37) u.  All of that of sum p|v|;
  * a weight of a row below 2^-126 may be lost, in three terms, as may those bits of it: a weight is in units of up to twice
    the largest scale (a code of which is that of up to the largest value), so n 2^-123 max|v| at most;
  * a result below 2^-126 may be 0: for the 80 items and lanes' sums that are added at most, 2^-119;
  * and half a step of the output's type."""
import math

import numpy as np
import pytest
import torch

import paper_2511_03092_amd as snap
from blockhelp import Blocks, choose, params
from pagedhelp import HALF_STEP, U
from test_gpu_blocks import _call, _i32, _load, _rand

pytestmark = pytest.mark.gpu


def _rows_of(c, slot, g, r, q, max_rows, select):
    """Keys and values [n, d] in float64 that the heads of group g attend, newest row r."""
    p, B = c.p, c.block
    n, T, G = min(r, max_rows) // B, r // B, p.n_q_heads // p.n_kv_heads
    blocks = choose(c, slot, g, r, q[g * G:(g + 1) * G].cpu(), max_rows) if select else list(range(n))
    return [torch.cat((c.values(x, slot, g, blocks), c.x[x][slot][T * B:r + 1, g].double())).numpy() for x in ("k", "v")]


def _check(c, slots, rows, q, out, select=False):
    p = c.p
    G, d = p.n_q_heads // p.n_kv_heads, p.d_qk
    scale = p.sm_scale if p.sm_scale > 0 else 1.0 / math.sqrt(d)
    for b, (slot, r) in enumerate(zip(slots, rows)):
        for g in range(p.n_kv_heads):
            k, v = _rows_of(c, slot, g, r, q[b], c.max_pages * c.page, select)
            n = len(k)
            for h in range(g * G, (g + 1) * G):
                qh = q[b, h].double().cpu().numpy()
                z = scale * (k @ qh)
                dz = scale * (d + 4) * U * np.abs(k * qh).sum(1).max()
                e = np.exp(z - z.max())
                pr = e / e.sum()
                want = pr @ v
                err = (2 * dz + (64 + 16 + 2 * (n / 32 + 37)) * U) * (pr @ np.abs(v)) + n * 2.0 ** -123 * np.abs(v).max() + 2.0 ** -119
                got = out[b, h].double().cpu().numpy()
                tol = err + HALF_STEP[out.dtype] * (np.abs(want) + err)
                off = np.abs(got - want)
                assert (off <= tol).all(), (b, h, n, (off / tol).max(), (off / np.abs(want)).max())


@pytest.mark.parametrize("factor", [1e-18, 1e-24, 1e-30, 1e30])
@pytest.mark.parametrize("kv,d,block,page", [("i8", 64, 32, 64), ("i8", 128, 64, 64), ("fp8", 64, 64, 128), ("fp8", 128, 32, 32),
                                             ("bf16", 64, 32, 32), ("bf16", 128, 64, 128)])
def test_values_of_every_size_keep_fp32_errors(kv, d, block, page, factor):
    """Small logits, so that the bound is a few hundred u; values of one sign, so that what is added shows.  300 rows by one
    launch, 9000 by two, and some of their blocks."""
    print(f"\n[case] {kv} d {d} block {block}: values times {factor}", flush=True)
    p = params(4, 2, d, kv, sink=4, recent=200, topk=900)
    lengths = [300, 9000, 33]
    c = Blocks(p, kv, block, page, lengths, 1)
    g = torch.Generator().manual_seed(2)
    k = _rand(g, 3, 2, 9000, d)
    v = ((0.05 + _rand(g, 3, 2, 9000, d).float().abs()) * factor).bfloat16()
    _load(c, [0, 1, 2], lengths, 3, like=(k, v))
    c.rows -= 1
    q = (_rand(g, 3, 4, d, spread=False).float() / 16).bfloat16().cuda()
    for slots in ([0], [0, 1, 2]):
        rows, qs = [lengths[s] - 1 for s in slots], q[:len(slots)]
        for select in (False, True):
            out, _ = _call(c, slots, qs, max_rows=300 if slots == [0] else None, select=select, dtype=torch.float32)
            _check(c, slots, rows, qs, out, select)
    new = [x.cuda() for x in (k[:, :, :1].contiguous(), v[:, :, :1].contiguous())]
    out, _ = _call(c, [0, 1, 2], q, new=new)  # a step: the last row once more
    for s, n in enumerate(lengths):
        for name, x in (("k", k), ("v", v)):
            c.x[name][s][n - 1] = x[s, :, 0]
    if kv == "bf16":  # (8 bits: the last rows are no whole block's)
        _check(c, [0, 1, 2], [n - 1 for n in lengths], q, out)


@pytest.mark.parametrize("kv", ["i8", "fp8", "bf16"])
@pytest.mark.parametrize("spread", [10, 30])
def test_blocks_of_unequal_size(kv, spread):
    """Each block's values times a power of ten of its own, up to 10^+-spread."""
    print(f"\n[case] {kv}: values of blocks from 1e-{spread} to 1e{spread}", flush=True)
    p = params(4, 2, 64, kv)
    lengths = [400, 6000]
    c = Blocks(p, kv, 32, 64, lengths, 1, bounds=False)
    g = torch.Generator().manual_seed(4)
    size = 10.0 ** (spread * (2 * torch.rand((2, 2, 6016 // 32, 1, 1), generator=g) - 1))
    k = _rand(g, 2, 2, 6000, 64)
    v = ((0.05 + _rand(g, 2, 2, 6016, 64).float().abs()).unflatten(2, (-1, 32)) * size).flatten(2, 3)[:, :, :6000].bfloat16()
    _load(c, [0, 1], lengths, 3, like=(k, v))
    c.rows -= 1
    q = (_rand(g, 2, 4, 64, spread=False).float() / 16).bfloat16().cuda()
    for slots in ([0], [0, 1]):
        out, _ = _call(c, slots, q[:len(slots)], max_rows=400 if slots == [0] else None, dtype=torch.float32)
        _check(c, slots, [lengths[s] - 1 for s in slots], q[:len(slots)], out)


@pytest.mark.parametrize("whole,newest", [(1e-30, 1.0), (1e30, 1.0), (1.0, 1e-30), (1.0, 1e30), (1e-20, 1e15), (1e37, 1e-30)])
@pytest.mark.parametrize("kv,d", [("i8", 128), ("fp8", 64), ("bf16", 64)])
def test_the_newest_block_beside_blocks_of_another_size(kv, d, whole, newest):
    """A wave that goes from codes to rows as they came, and back to none; the newest block's rows with most of the sum, and
    with little of it."""
    print(f"\n[case] {kv} d {d}: whole blocks times {whole}, the newest times {newest}", flush=True)
    p = params(4, 2, d, kv, sm_scale=1.0)
    lengths = [300, 300, 45, 4127]
    c = Blocks(p, kv, 32, 64, lengths, 1, bounds=False)
    g = torch.Generator().manual_seed(8)
    k = (_rand(g, 4, 2, 4127, d, spread=False).float() / 16).bfloat16()
    v = 0.05 + _rand(g, 4, 2, 4127, d).float().abs()
    for b, n in enumerate(lengths):
        tail = slice((n - 1) // 32 * 32, n)
        v[b] *= whole
        v[b, :, tail] *= newest / whole
        k[b, :, tail, 5] = 4.0 if b % 2 else -4.0
    v = v.bfloat16()
    _load(c, [0, 1, 2, 3], lengths, 3, like=(k, v))
    c.rows -= 1
    q = (_rand(g, 4, 4, d, spread=False).float() / 16).bfloat16()
    q[..., 5] = 4.0
    q = q.cuda()
    for slots in ([0, 1, 2], [0, 1, 2, 3]):
        out, _ = _call(c, slots, q[:len(slots)], max_rows=300 if len(slots) == 3 else None, dtype=torch.float32)
        _check(c, slots, [lengths[s] - 1 for s in slots], q[:len(slots)], out)


@pytest.mark.parametrize("kv", ["i8", "fp8", "bf16"])
@pytest.mark.parametrize("big", [1e20, 1e30, 1e37])
@pytest.mark.parametrize("first", [True, False], ids=["first", "last"])
def test_rows_without_a_share_add_nothing(kv, big, first):
    """Blocks of large values whose probability is below any number beside blocks of ordinary ones, before and behind."""
    print(f"\n[case] {kv}: values of {big} in rows without a share", flush=True)
    p = params(2, 1, 64, kv, sm_scale=1.0)
    lengths = [420, 5000]
    c = Blocks(p, kv, 32, 64, lengths, 1, bounds=False)
    g = torch.Generator().manual_seed(5)
    k = (_rand(g, 2, 1, 5000, 64, spread=False).float() / 8).bfloat16()
    v = (0.05 + _rand(g, 2, 1, 5000, 64).float().abs()).bfloat16()
    for b, n in enumerate(lengths):  # a third of the whole blocks
        whole = (n - 1) // 32 // 3 * 32
        at = slice(0, whole) if first else slice((n - 1) // 32 * 32 - whole, (n - 1) // 32 * 32)
        k[b, :, at, 7] = -16.0
        v[b, :, at] = (v[b, :, at].float() * big).bfloat16()
    _load(c, [0, 1], lengths, 3, like=(k, v))
    c.rows -= 1
    q = (_rand(g, 2, 2, 64, spread=False).float() / 8).bfloat16()
    q[..., 7] = 16.0  # logits of -256 (nats) there, whatever the codes of the others
    q = q.cuda()
    for slots in ([0], [0, 1]):
        out, _ = _call(c, slots, q[:len(slots)], max_rows=420 if slots == [0] else None, dtype=torch.float32)
        for b, slot in enumerate(slots):  # the others alone
            for h in range(2):
                kk, vv = _rows_of(c, slot, 0, lengths[slot] - 1, q[b], 1 << 20, False)
                qh = q[b, h].double().cpu().numpy()
                z = kk @ qh
                assert z.max() - z[kk[:, 7] < -8].max() > 150
                keep = kk[:, 7] > -8
                dz = 68 * U * np.abs(kk[keep] * qh).sum(1).max()
                e = np.exp(z[keep] - z.max())
                pr = e / e.sum()
                want, n = pr @ vv[keep], len(kk)
                # z up to 64 or so beside them; weights below 2^-126 in units of these rows' scales
                err = (2 * dz + (64 + 16 + 2 * (n / 32 + 37)) * U) * (pr @ np.abs(vv[keep])) + n * 2.0 ** -110
                got = out[b, h].double().cpu().numpy()
                tol = err + HALF_STEP[out.dtype] * (np.abs(want) + err)
                assert (np.abs(got - want) <= tol).all(), (slot, h, (np.abs(got - want) / tol).max(), np.abs(got - want).max())


@pytest.mark.parametrize("kv,d,block,page", [("i8", 128, 64, 64), ("fp8", 64, 32, 64), ("bf16", 128, 64, 128), ("bf16", 64, 32, 32),
                                             ("i8", 64, 128, 128), ("fp8", 128, 64, 64)])
@pytest.mark.parametrize("length", [300, 3000])
def test_probabilities_lose_no_bits_before_the_values(kv, d, block, page, length):
    """Values that are all one, so that their weighted mean is: the first row of every 32 has logit 0, the others the one
    whose exp is half of 1 + 2^-7 - 2^-17, which two terms of 8 bits, cut off, would miss by 2^-15 - 2^-17, 384 u.  The same
    probabilities are in the product and in the sum below it, so that logits and exp2 have no part in the error."""
    print(f"\n[case] {kv} d {d} block {block}, {length} rows, values all one", flush=True)
    p = params(4, 2, d, kv)
    c = Blocks(p, kv, block, page, [length], 1, bounds=False)
    k = torch.zeros((1, 2, length, d), dtype=torch.bfloat16)
    k[..., d - 3:] = 1.0
    k[:, :, ::32] = 0.0
    _load(c, [0], [length], 1, like=(k, torch.ones_like(k)))
    c.rows -= 1
    rest = math.log(0.5 * (1 + 2.0 ** -7 - 2.0 ** -17)) * math.sqrt(d)
    q = torch.zeros((1, 4, d), dtype=torch.bfloat16)
    for i in range(3):  # to 24 bits
        q[..., d - 3 + i] = rest
        rest -= float(q[0, 0, d - 3 + i])
    for mr in (length, page * c.max_pages):
        out, _ = _call(c, [0], q.cuda(), max_rows=mr, dtype=torch.float32)
        # an item has all steps at most; 2 u: a code times its block's scale is one but for them
        tol = (2 * (length / 32 + 37) + 16 + 2) * U
        err = float((out.double() - 1).abs().max())
        assert err <= tol, (err / U, tol / U)


@pytest.mark.parametrize("kv,d,block", [("i8", 128, 64), ("fp8", 64, 32), ("bf16", 128, 64), ("bf16", 64, 32)])
@pytest.mark.parametrize("length", [20, 300, 5000, 70000])
@pytest.mark.parametrize("rising", [False, True], ids=["any", "rising"])
def test_the_largest_values_stay_finite(kv, d, block, length, rising):
    """Every value is the largest of bf16, of either sign by its dim; logits in any order, or rising by less than what the
    reference lags behind for many rows at a time (e^5 within 2^8)."""
    print(f"\n[case] {kv} d {d} block {block}, {length} rows of the largest value, rising {rising}", flush=True)
    p = params(2, 1, d, kv, sm_scale=1.0)
    c = Blocks(p, kv, block, 128, [length], 1, bounds=False)
    g = torch.Generator().manual_seed(9)
    k = (_rand(g, 1, 1, length, d, spread=False).float() / 16).bfloat16()
    if rising:
        k[0, 0, :, 0] = 5.0 * torch.arange(length) / length
    v = torch.full((1, 1, length, d), torch.finfo(torch.bfloat16).max, dtype=torch.bfloat16)
    v[..., ::2] *= -1
    _load(c, [0], [length], 1, like=(k, v))
    c.rows -= 1
    q = (_rand(g, 1, 2, d, spread=False).float() / 16).bfloat16()
    q[..., 0] = 1.0
    for dtype in (torch.float32, torch.bfloat16):
        out, _ = _call(c, [0], q.cuda(), max_rows=length, dtype=dtype)
        rel = (out.double().cpu() / v[0, 0, 0].double() - 1).abs()
        # as for values of one: the same probabilities in both sums, 18 u beside the additions
        assert float(rel.max()) <= (2 * (length / 32 + 37) + 18) * U + (0.0 if dtype == torch.float32 else 2.0 ** -8)


@pytest.mark.parametrize("newest", [False, True], ids=["codes", "newest"])
@pytest.mark.parametrize("length", [84, 2000])
@pytest.mark.parametrize("kv,d,block", [("i8", 128, 64), ("fp8", 64, 64), ("bf16", 128, 64), ("i8", 64, 32), ("fp8", 128, 32),
                                        ("bf16", 64, 32)])
def test_two_terms_of_a_probability_would_show(kv, d, block, length, newest):
    """Nine rows of one 32-row step share the softmax: one of logit 0 and eight whose probability beside it is half of
    1 + 2^-9 + 2^-17 - 2^-21.  Two terms of 8 bits, cut off or rounded to nearest, miss that by 2^-17 - 2^-21, 120 u, in eight
    of ten parts of the sum: 96 u.  Nine terms have eight additions that are not of zeros, in each sum: with 18 u as above
    34 u.  Values are the type's largest code, whose scale is one to a rounding."""
    print(f"\n[case] {kv} d {d} block {block}, nine of {length} rows, newest {newest}", flush=True)
    p = params(4, 2, d, kv)
    c = Blocks(p, kv, block, block, [length], 1, bounds=False)
    top = {"i8": 127.0, "fp8": 448.0, "bf16": 1.0}[kv]
    k = torch.zeros((1, 2, length, d), dtype=torch.bfloat16)
    k[..., d - 4] = 1.0  # without a share
    at = (length - 1) // 32 * 32 if newest else length // 2 // 32 * 32
    assert newest == (at >= (length - 1) // block * block) and at + 9 <= length
    k[:, :, at:at + 9, d - 4] = 0.0
    k[:, :, at + 1:at + 9, d - 3:] = 1.0
    _load(c, [0], [length], 1, like=(k, torch.full_like(k, top)))
    c.rows -= 1
    rest = math.log(0.5 * (1 + 2.0 ** -9 + 2.0 ** -17 - 2.0 ** -21)) * math.sqrt(d)
    q = torch.zeros((1, 4, d), dtype=torch.bfloat16)
    q[..., d - 4] = -300.0 * math.sqrt(d)
    for i in range(3):  # to 24 bits
        q[..., d - 3 + i] = rest
        rest -= float(q[0, 0, d - 3 + i])
    out, _ = _call(c, [0], q.cuda(), max_rows=length, dtype=torch.float32)
    err = float((out.double() / top - 1).abs().max())
    assert err <= 34 * U, err / U


# ---------------------------------------------------------------- infinities and NaN
def _special(kv, length, marks, select=False, keys=(), newest=()):
    """Attention with single values (row, dim, what) and keys replaced, outputs and the definition's in float64."""
    p = params(4, 2, 64, kv, sm_scale=0.125, sink=4, recent=100, topk=10000)
    c = Blocks(p, kv, 32, 64, [length], 1)
    g = torch.Generator().manual_seed(6)
    k, v = _rand(g, 1, 2, length, 64, spread=False), _rand(g, 1, 2, length, 64, spread=False)
    q = _rand(g, 1, 4, 64, spread=False)
    q[:] = torch.where(q.abs() < 0.1, torch.full_like(q, 0.5), q)
    for r, i, x in marks:
        v[0, 0, r, i] = x
    for r, i, x in keys:
        k[0, 0, r, i] = x
    _load(c, [0], [length], 1, like=(k, v))
    c.rows -= 1
    out, _ = _call(c, [0], q.cuda(), max_rows=length, select=select, dtype=torch.float32)
    kk, vv = (torch.cat((c.values(n, 0, 0, range((length - 1) // 32)), c.x[n][0][(length - 1) // 32 * 32:, 0].double()))
              for n in ("k", "v"))
    z = 0.125 * (q[0, :2].double() @ kk.T.contiguous())
    want = torch.softmax(z, -1)[:, :, None] * vv[None]
    return out[0, :2].double().cpu(), want.sum(1), out[0, 2:]


def _alike(got, want):
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (got, want)
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], want[inf])
    ok = torch.isfinite(want)
    assert float((got[ok] - want[ok]).abs().max() if ok.any() else 0.0) <= 1e-3  # (the dims beside them)


@pytest.mark.parametrize("select", [False, True], ids=["all", "select"])
@pytest.mark.parametrize("length", [200, 2100])
@pytest.mark.parametrize("kv", ["bf16", "i8", "fp8"])
def test_infinite_and_nan_values(kv, length, select):
    """In rows that are read as they came they are infinite or NaN in their dim of the heads that share them, and in no
    other; codes of 8 bits hold no infinity, and a NaN in E4M3 alone."""
    print(f"\n[case] {kv}: infinite and NaN values among {length} rows, select {select}", flush=True)
    inf, nan = math.inf, math.nan
    r = length - 1 if kv != "bf16" else 40
    marks = [(r, 3, inf), (r, 5, -inf), (r, 9, nan), (length - 1, 20, inf)]
    if kv == "bf16":
        marks += [(0, 30, inf), (77, 30, inf), (0, 31, inf), (150, 31, -inf)]
    else:
        marks += [(40, 40, inf), (41, 41, nan)]
    got, want, others = _special(kv, length, marks, select)
    assert torch.isfinite(others).all()
    if kv != "bf16":  # (clamped to the block's largest code; a NaN is 0 in int8)
        assert torch.isfinite(want[:, 40]).all() and torch.isnan(want[:, 41]).all() == (kv == "fp8")
    _alike(got, want)


@pytest.mark.parametrize("length", [200, 2100])
@pytest.mark.parametrize("kv", ["bf16", "i8", "fp8"])
def test_infinite_and_nan_keys(kv, length):
    """A key with -infinity times a positive number has no share; one with a NaN makes the heads that attend it NaN, but in
    the codes of int8, where it is 0."""
    print(f"\n[case] {kv}: infinite and NaN keys among {length} rows", flush=True)
    nan, r = math.nan, length - 1
    for at in (40, r):
        got, want, others = _special(kv, length, [], keys=[(at, 3, nan)])
        assert torch.isfinite(others).all()
        if kv == "i8" and at == 40:
            assert torch.isfinite(want).all()
        else:
            assert torch.isnan(want).all()
        _alike(got, want)
    for at in (40, r):  # (the heads' signs differ: -inf for one is +inf, so NaN, for another)
        got, want, others = _special(kv, length, [], keys=[(at, 3, -math.inf)])
        assert torch.isfinite(others).all()
        _alike(got, want)


@pytest.mark.parametrize("length", [200, 2100])
def test_an_infinite_value_without_a_share_is_no_number_less(length):
    """Where a row's share is below what fp32 holds its infinity stays infinite or gives NaN, never a finite number."""
    print(f"\n[case] an infinite value in a row without a share, {length} rows", flush=True)
    p = params(2, 1, 64, "bf16", sm_scale=1.0)
    c = Blocks(p, "bf16", 32, 64, [length], 1, bounds=False)
    g = torch.Generator().manual_seed(7)
    k, v = _rand(g, 1, 1, length, 64, spread=False), _rand(g, 1, 1, length, 64, spread=False)
    k[..., 0] = 0.0
    k[0, 0, 50, 0], k[0, 0, 51, 0], k[0, 0, 52, 0], k[0, 0, 53, 0] = -40.0, -16.0, -1.5, -6.0
    v[0, 0, 50, 1], v[0, 0, 51, 2], v[0, 0, 52, 3], v[0, 0, 53, 0] = math.inf, math.inf, -math.inf, math.inf
    _load(c, [0], [length], 1, like=(k, v))
    c.rows -= 1
    q = torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    q[..., 0] = 8.0
    out, _ = _call(c, [0], q.cuda(), max_rows=length, dtype=torch.float32)
    out = out[0].cpu()
    assert not torch.isfinite(out[:, 1]).any() and not torch.isfinite(out[:, 2]).any()
    assert (out[:, 3] == -math.inf).all() and (out[:, 0] == math.inf).all()  # shares of e^-12 and e^-48 beside rows of one
    assert torch.isfinite(out[:, 4:]).all()
