"""Refusals of the rotary and paged calls: every one is decided on the host before anything would be launched, so these
run without a GPU."""
import ctypes

import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import params

FAKE = 0x100000  # aligned, never dereferenced (validation fails first)
INVALID, UNSUPPORTED, WORKSPACE = snap.SNAP_ERR_INVALID_ARG, snap.SNAP_ERR_UNSUPPORTED, snap.SNAP_ERR_WORKSPACE


def _heads(x=FAKE, y=FAKE + (1 << 20), xs=(2048, 512, 64), ys=(2048, 512, 64), heads=4):
    i3 = ctypes.c_int64 * 3
    return snap.SnapRopeHeads(x, y, i3(*xs), i3(*ys), heads)


def _rope(r=None, dtype=snap.SNAP_BF16, n=2, tokens=8, d=64, pos=None, n_slots=0, slots=None, q=None, k=None, null=False):
    r = r or snap.RopeParams(0, 64)
    L = snap.lib()
    q = _heads() if q is None else q
    st = L.snap_rope(None if null else ctypes.byref(r.c()), dtype, n, tokens, d, pos, n_slots, slots, None,
                     ctypes.byref(q), None if k is None else ctypes.byref(k), None)
    return st, L.snap_last_error().decode()


R = snap.RopeParams


@pytest.mark.parametrize("kw,code", [
    (dict(null=True), INVALID),
    (dict(dtype=snap.SNAP_FP8_E4M3), INVALID),
    (dict(r=R(0, 63)), INVALID),
    (dict(r=R(0, 0)), INVALID),
    (dict(r=R(0, 130), d=256), INVALID),
    (dict(r=R(2, 64)), INVALID),
    (dict(r=R(-2, 64)), INVALID),
    (dict(r=R(0, 64, layout=2)), INVALID),
    (dict(r=R(0, 64, rule=4)), INVALID),
    (dict(r=R(0, 64, base=1.0)), INVALID),
    (dict(r=R(0, 64, base=float("nan"))), INVALID),
    (dict(r=R(0, 64, amplitude=0.0)), INVALID),
    (dict(r=R(0, 64, rule=snap.SNAP_ROPE_DIVIDE, factor=0.5)), INVALID),
    (dict(r=R(0, 64, rule=snap.SNAP_ROPE_BY_TURNS, low_turns=4.0, high_turns=4.0, orig_len=10)), INVALID),
    (dict(r=R(0, 64, rule=snap.SNAP_ROPE_BY_INDEX, low_turns=0.0, orig_len=10)), INVALID),
    (dict(r=R(0, 64, rule=snap.SNAP_ROPE_BY_TURNS, orig_len=0)), INVALID),
    (dict(n=-1), INVALID),
    (dict(tokens=0), INVALID),
    (dict(n=1 << 20, tokens=1 << 10), UNSUPPORTED),
    (dict(d=1), INVALID),
    (dict(pos=FAKE), INVALID),
    (dict(pos=FAKE, slots=FAKE), INVALID),
    (dict(q=_heads(x=0)), INVALID),
    (dict(q=_heads(y=0)), INVALID),
    (dict(q=_heads(x=FAKE + 1)), INVALID),
    (dict(q=_heads(heads=0)), INVALID),
    (dict(q=_heads(ys=(2048, 512, 0))), INVALID),
    (dict(q=_heads(y=FAKE + 64)), INVALID),
    (dict(q=_heads(y=FAKE, ys=(2048, 64, 256))), INVALID),
    (dict(q=_heads(y=FAKE + 8192, ys=(-2048, 512, 64))), INVALID),
    (dict(q=_heads(xs=(1 << 62, 512, 64))), INVALID),
    (dict(k=_heads(heads=0)), INVALID),
    (dict(k=_heads(y=FAKE + 2)), INVALID),
])
def test_rope_refusals(kw, code):
    st, msg = _rope(**kw)
    assert st == code and msg


def test_no_sequences_is_a_no_op():
    assert _rope(n=0)[0] == snap.SNAP_OK
    p = params(8, 2, 64)
    c = snap.SnapPagedCache(FAKE, FAKE, None, None, FAKE, FAKE, FAKE, 4, 10, 16, 8)
    L, P, C = snap.lib(), ctypes.byref(p.c()), ctypes.byref(c)
    assert L.snap_paged_append(P, C, FAKE, FAKE, 0, FAKE, None, 1, FAKE, None, FAKE, None, None, None) == 0
    assert L.snap_paged_decode_attn(P, C, FAKE, 0, FAKE, 10, FAKE, FAKE, 1, 0, None, 0, None) == 0
    assert L.snap_paged_decode_step(P, C, FAKE, FAKE, 0, FAKE, 10, FAKE, FAKE, FAKE, FAKE, 1, 0, None, 0, None) == 0
    assert L.snap_paged_evict(P, C, FAKE, FAKE, FAKE, 0, FAKE, 10, None, None, 0, None) == 0


CACHE = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, token=FAKE, weight=FAKE, page_table=FAKE, n_slots=4, n_pages=10,
             page_size=16, max_pages=8)


def _calls(pkw=None, ckw=None, **kw):
    """Status and message of append, attention, step and eviction with one argument wrong."""
    pkw = dict(pkw or {})
    p = params(pkw.pop("hq", 8), pkw.pop("hkv", 2), pkw.pop("d", 64), pkw.pop("kv", "bf16"), pkw.pop("latent", False), **pkw)
    a = dict(rows=FAKE, pos=FAKE, n=2, slots=FAKE, max_len=4, max_rows=100, k_new=FAKE, v_new=None if p.v_in_k else FAKE,
             ks=None, q=FAKE, out=FAKE, od=1, weigh=1, ws=FAKE, size=1 << 40, rows_out=FAKE + 64)
    a.update(kw)
    c = snap.SnapPagedCache(**{**CACHE, **({"v": None} if p.v_in_k else {}), **(ckw or {})})
    L, P, C = snap.lib(), ctypes.byref(p.c()), ctypes.byref(c)
    got = {}

    def call(name, fn, *args):
        st = fn(*args)
        got[name] = (st, L.snap_last_error().decode())

    ks = None if a["ks"] is None else (ctypes.c_int64 * 3)(*a["ks"])
    if "append" in kw.get("only", "append"):
        call("append", L.snap_paged_append, P, C, a["rows"], a["pos"], a["n"], a["slots"], None, a["max_len"], a["k_new"],
             ks, a["v_new"], None, None, None)
    if "attn" in kw.get("only", "attn"):
        call("attn", L.snap_paged_decode_attn, P, C, a["rows"], a["n"], a["slots"], a["max_rows"], a["q"], a["out"],
             a["od"], a["weigh"], a["ws"], a["size"], None)
    if "step" in kw.get("only", "step"):
        call("step", L.snap_paged_decode_step, P, C, a["rows"], a["pos"], a["n"], a["slots"], a["max_rows"], a["q"],
             a["k_new"], a["v_new"], a["out"], a["od"], a["weigh"], a["ws"], a["size"], None)
    if "evict" in kw.get("only", "evict"):
        call("evict", L.snap_paged_evict, P, C, a["rows"], a["pos"], a["rows_out"], a["n"], a["slots"], a["max_rows"],
             None, a["ws"], a["size"], None)
    return got


ALL = "append attn step evict"


@pytest.mark.parametrize("kw,code,only", [
    (dict(pkw=dict(hq=7)), INVALID, ALL),
    (dict(pkw=dict(d=96)), UNSUPPORTED, ALL),
    (dict(pkw=dict(d=128, kv="fp8", fp8_qk=1), ckw=dict(k_scale=FAKE, v_scale=FAKE)), UNSUPPORTED, ALL),
    (dict(ckw=dict(k=None)), INVALID, ALL),
    (dict(ckw=dict(v=None)), INVALID, ALL),
    (dict(ckw=dict(k=FAKE + 8)), INVALID, ALL),
    (dict(ckw=dict(page_table=None)), INVALID, ALL),
    (dict(ckw=dict(weight=FAKE + 4)), INVALID, ALL),
    (dict(ckw=dict(token=FAKE + 8)), INVALID, ALL),
    (dict(ckw=dict(n_slots=0)), INVALID, ALL),
    (dict(ckw=dict(n_pages=0)), INVALID, ALL),
    (dict(ckw=dict(max_pages=0)), INVALID, ALL),
    (dict(ckw=dict(page_size=8)), UNSUPPORTED, ALL),
    (dict(ckw=dict(page_size=48)), UNSUPPORTED, ALL),
    (dict(ckw=dict(page_size=8192)), UNSUPPORTED, ALL),
    (dict(ckw=dict(max_pages=1 << 25)), INVALID, ALL),
    (dict(pkw=dict(kv="fp8")), INVALID, ALL),
    (dict(n=-1), INVALID, ALL),
    (dict(n=40000), UNSUPPORTED, ALL),
    (dict(rows=None), INVALID, ALL),
    (dict(slots=None), INVALID, ALL),
    (dict(pos=None), INVALID, "append step evict"),
    (dict(k_new=None), INVALID, "append step"),
    (dict(k_new=FAKE + 4), INVALID, "append step"),
    (dict(v_new=None), INVALID, "append step"),
    (dict(max_len=0), INVALID, "append"),
    (dict(max_len=(1 << 28) + 1), INVALID, "append"),
    (dict(ks=(512, 64, 12)), INVALID, "append"),
    (dict(max_rows=0), INVALID, "attn step evict"),
    (dict(max_rows=129), INVALID, "attn step evict"),
    (dict(q=None), INVALID, "attn step"),
    (dict(out=FAKE + 2), INVALID, "attn step"),
    (dict(od=2), INVALID, "attn step"),
    (dict(weigh=2), INVALID, "attn step"),
    (dict(ckw=dict(weight=None)), INVALID, "attn step evict"),
    (dict(ckw=dict(token=None)), INVALID, "evict"),
    (dict(rows_out=None), INVALID, "evict"),
    (dict(rows_out=FAKE), INVALID, "evict"),
    (dict(ws=None), WORKSPACE, "attn step evict"),
    (dict(ws=FAKE + 16), WORKSPACE, "attn step evict"),
    (dict(size=64), WORKSPACE, "attn step evict"),
])
def test_paged_refusals(kw, code, only):
    for name, (st, msg) in _calls(only=only, **kw).items():
        assert st == code and msg, (name, st, msg)


def test_workspace_queries():
    p = params(32, 8, 128)
    a = snap.snap_paged_decode_workspace(p, 4, 10000)
    assert a > 0 and snap.snap_paged_decode_workspace(p, 4, 10000, True) >= a + 4 * 32 * 10000 * 4
    assert snap.snap_paged_decode_workspace(p, 4, 0) == 0 and snap.snap_paged_decode_workspace(p, -1, 10) == 0
    assert snap.snap_paged_decode_workspace(p, 4, (1 << 28) + 1) == 0
    assert snap.snap_paged_evict_workspace(p, 4, 10000) > 0 and snap.snap_paged_evict_workspace(p, 4, 0) == 0
    assert snap.snap_paged_evict_workspace(params(7, 2, 64), 4, 100) == 0


def test_binding_refuses_tensors_that_do_not_fit():
    """What the library cannot see: types, shapes, strides, devices."""
    p = params(8, 2, 64)
    k = torch.zeros((10, 2, 16, 64), dtype=torch.bfloat16)
    table, ids, rows = (torch.zeros(s, dtype=torch.int32) for s in ((4, 8), (2,), (4,)))
    c = snap.paged_cache_struct(k, k.clone(), table, torch.zeros((10, 2, 16), dtype=torch.int32), torch.zeros((10, 2, 16)))
    new, q = torch.zeros((2, 2, 1, 64), dtype=torch.bfloat16), torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    out, ws = torch.zeros_like(q), torch.zeros(1 << 20, dtype=torch.uint8)
    bad = [
        lambda: snap.paged_cache_struct(k[:, :, ::2], k, table),
        lambda: snap.paged_cache_struct(k, k[:5], table),
        lambda: snap.paged_cache_struct(k, k.float(), table),
        lambda: snap.paged_cache_struct(k, k, table.long()),
        lambda: snap.paged_cache_struct(k, k, table, token=torch.zeros((10, 2, 16))),
        lambda: snap.paged_cache_struct(k, k, table, weight=torch.zeros((10, 16, 2))),
        lambda: snap.paged_cache_struct(k.half(), k, table),
        lambda: snap.snap_paged_append(params(8, 4, 64), c, rows, rows, ids, new, new),
        lambda: snap.snap_paged_append(params(8, 2, 64, "f32"), c, rows, rows, ids, new, new),
        lambda: snap.snap_paged_append(p, c, rows.long(), rows, ids, new, new),
        lambda: snap.snap_paged_append(p, c, rows[:3], rows, ids, new, new),
        lambda: snap.snap_paged_append(p, c, rows, rows, ids, new, None),
        lambda: snap.snap_paged_append(p, c, rows, rows, ids, new.float(), new),
        lambda: snap.snap_paged_append(p, c, rows, rows, ids, new.transpose(2, 3), new),
        lambda: snap.snap_paged_append(p, c, rows, rows, ids, new, new, lengths=ids.long()),
        lambda: snap.snap_paged_append(p, c, rows, rows, ids, new, new, weight_new=torch.zeros((2, 2, 2))),
        lambda: snap.snap_paged_decode_attn(p, c, rows, ids, q[:, :4], out, ws),
        lambda: snap.snap_paged_decode_attn(p, c, rows, ids, q, out.half(), ws),
        lambda: snap.snap_paged_decode_step(p, c, rows, rows, ids, q, new, None, out, ws),
        lambda: snap.snap_paged_decode_step(p, c, rows, rows, ids, q, new[:1], new, out, ws),
        lambda: snap.snap_paged_evict(p, c, rows, None, ids, rows, ws),
        lambda: snap.snap_paged_evict(p, c, rows, rows, ids, rows, ws, kept_out=torch.zeros((2, 2, 3), dtype=torch.int32)),
        lambda: snap.snap_paged_append(p, c, rows, rows, ids, new, new),  # not on the GPU
        lambda: snap.snap_rope(R(0, 64), new.transpose(2, 3)),
        lambda: snap.snap_rope(R(0, 64), new.half()),
        lambda: snap.snap_rope(R(0, 64), new, new[:1]),
        lambda: snap.snap_rope(R(0, 64), new, new.float()),
        lambda: snap.snap_rope(R(0, 64), new, q_out=new[:, :1]),
        lambda: snap.snap_rope(R(0, 64), new, pos=rows, slot_ids=ids.long()),
        lambda: snap.snap_rope(R(0, 64), new, pos=rows),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(snap.SnapError) as e:
            f()
        assert e.value.status == INVALID, i
