"""Refusals of the page-table, mapped and block calls: every one is decided on the host before anything would be launched,
so these run without a GPU."""
import ctypes

import pytest
import torch

import paper_2511_03092_amd as snap
import pagedhelp
from blockhelp import params

FAKE = 0x100000  # aligned, never dereferenced (validation fails first)
INVALID, UNSUPPORTED, WORKSPACE = snap.SNAP_ERR_INVALID_ARG, snap.SNAP_ERR_UNSUPPORTED, snap.SNAP_ERR_WORKSPACE
BIG = 1 << 40


def _cache(**kw):
    a = {n: FAKE for n in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail", "bound", "bound_scale", "page_table")}
    a.update(n_slots=8, n_pages=100, page_size=64, max_pages=16, block=32)
    a.update(kw)
    return snap.SnapBlockCache(**a)


def _pool(**kw):
    a = dict(page_table=FAKE, held=FAKE, free_pages=FAKE, n_free=FAKE, n_slots=8, n_pages=100, page_size=64, max_pages=16)
    a.update(kw)
    return snap.SnapPagePool(**a)


def _run(call, p, c, a):
    L, P, C = snap.lib(), ctypes.byref(p.c()), ctypes.byref(c)
    if call == "append":
        st = L.snap_block_append(P, C, a["rows"], a["n"], a["slots"], a["lengths"], a["starts"], a["tokens"], a["max_len"], a["k_new"],
                                 a["k_stride"], a["v_new"], a["v_stride"], None)
    elif call == "attn":
        st = L.snap_block_decode_attn(P, C, a["rows"], a["n"], a["slots"], a["max_rows"], a["q"], a["out"], a["out_dtype"],
                                      a["select"], None, a["ws"], a["ws_bytes"], None)
    else:
        st = L.snap_block_decode_step(P, C, a["rows"], a["n"], a["slots"], a["max_rows"], a["q"], a["k_new"], a["v_new"], a["out"],
                                      a["out_dtype"], a["select"], None, a["ws"], a["ws_bytes"], None)
    return st, L.snap_last_error().decode()


ARGS = dict(rows=FAKE, n=2, slots=FAKE, lengths=None, starts=None, tokens=0, max_len=4, k_new=FAKE, k_stride=None, v_new=FAKE,
            v_stride=None, max_rows=512, q=FAKE, out=FAKE, out_dtype=snap.SNAP_BF16, select=0, ws=FAKE, ws_bytes=BIG)
I3 = ctypes.c_int64 * 3
ALL = ("append", "attn", "step")


@pytest.mark.parametrize("calls,p,c,a,code", [
    (ALL, dict(fp8_qk=1, kv="fp8", d=128), {}, {}, UNSUPPORTED),
    (ALL, dict(in_dtype=snap.SNAP_F32), {}, {}, UNSUPPORTED),
    (ALL, dict(kv_dtype=snap.SNAP_F32), {}, {}, UNSUPPORTED),
    (ALL, dict(kv_dtype=7), {}, {}, UNSUPPORTED),
    (ALL, dict(d_qk=576, d_v=512, v_in_k=True), {}, {}, UNSUPPORTED),
    (ALL, dict(hq=34), {}, {}, UNSUPPORTED),
    (ALL, dict(hq=5), {}, {}, INVALID),
    (ALL, dict(sm_scale=float("nan")), {}, {}, INVALID),
    (ALL, dict(recent=0), {}, {}, INVALID),
    (ALL, {}, dict(n_slots=0), {}, INVALID),
    (ALL, {}, dict(n_pages=0), {}, INVALID),
    (ALL, {}, dict(max_pages=0), {}, INVALID),
    (ALL, {}, dict(block=16), {}, UNSUPPORTED),
    (ALL, {}, dict(block=48), {}, UNSUPPORTED),
    (ALL, {}, dict(block=256, page_size=256), {}, UNSUPPORTED),
    (ALL, {}, dict(block=128), {}, UNSUPPORTED),
    (ALL, {}, dict(page_size=96), {}, UNSUPPORTED),
    (ALL, {}, dict(page_size=8192), {}, UNSUPPORTED),
    (ALL, {}, dict(max_pages=(1 << 22) + 1), {}, INVALID),
    (ALL, {}, dict(n_pages=0x7fffffff), {}, UNSUPPORTED),
    (ALL, {}, dict(page_table=None), {}, INVALID),
    (ALL, {}, dict(k=None), {}, INVALID),
    (ALL, {}, dict(v=FAKE + 8), {}, INVALID),
    (ALL, {}, dict(k_scale=None), {}, INVALID),
    (ALL, {}, dict(v_tail=None), {}, INVALID),
    (ALL, {}, dict(k_tail=FAKE + 2), {}, INVALID),
    (ALL, {}, dict(bound=None), {}, INVALID),
    (ALL, {}, dict(bound_scale=None), {}, INVALID),
    (ALL, {}, dict(bound=FAKE + 4), {}, INVALID),
    (ALL, {}, {}, dict(n=-1), INVALID),
    (ALL, {}, {}, dict(rows=None), INVALID),
    (ALL, {}, {}, dict(slots=None), INVALID),
    (("append",), {}, {}, dict(n=40000), UNSUPPORTED),
    (("append",), {}, {}, dict(max_len=0), INVALID),
    (("append",), {}, {}, dict(max_len=(1 << 28) + 1), INVALID),
    (("append",), {}, {}, dict(starts=FAKE, lengths=FAKE), INVALID),
    (("append",), {}, {}, dict(starts=FAKE, tokens=-1), INVALID),
    (("append",), {}, {}, dict(k_stride=I3(1024, 512, 68)), INVALID),
    (("append",), {}, {}, dict(v_stride=I3(1022, 512, 64)), INVALID),
    (("append", "step"), {}, {}, dict(k_new=None), INVALID),
    (("append", "step"), {}, {}, dict(v_new=FAKE + 8), INVALID),
    (("attn", "step"), {}, {}, dict(n=20000), UNSUPPORTED),
    (("attn", "step"), {}, {}, dict(max_rows=0), INVALID),
    (("attn", "step"), {}, {}, dict(max_rows=1025), INVALID),
    (("attn", "step"), {}, {}, dict(q=None), INVALID),
    (("attn", "step"), {}, {}, dict(out=FAKE + 4), INVALID),
    (("attn", "step"), {}, {}, dict(out_dtype=snap.SNAP_INT8), INVALID),
    (("attn", "step"), {}, {}, dict(select=2), INVALID),
    (("attn", "step"), {}, dict(bound=None, bound_scale=None), dict(select=1), INVALID),
    (("attn", "step"), {}, dict(page_size=4096, max_pages=1 << 16), dict(select=1, max_rows=32769 * 32), UNSUPPORTED),
    (("attn", "step"), {}, {}, dict(ws=None), WORKSPACE),
    (("attn", "step"), {}, {}, dict(ws=FAKE + 128), WORKSPACE),
    (("attn", "step"), {}, {}, dict(ws_bytes=1024), WORKSPACE),
])
def test_refusals_of_the_block_calls(calls, p, c, a, code):
    kw = dict(p)
    made = params(kw.pop("hq", 4), 2, kw.pop("d", 64), kw.pop("kv", "i8"), **kw)
    for call in calls:
        st, msg = _run(call, made, _cache(**c), {**ARGS, **a})
        assert st == code and msg, (call, st, msg)


def test_no_sequences_is_nothing_to_do():
    for call in ALL:
        assert _run(call, params(4, 2, 64), _cache(), {**ARGS, "n": 0, "rows": None, "ws": None, "ws_bytes": 0})[0] == snap.SNAP_OK


def test_int8_is_for_block_caches_alone():
    p = params(4, 2, 64, "i8")
    assert snap.snap_compress_workspace(p, 1, 100) == 0 and snap.snap_paged_decode_workspace(p, 1, 100) == 0
    assert snap.snap_block_decode_workspace(p, 1, 100, 32) > 0


def test_workspaces_do_not_fall():
    for kv, d in (("i8", 128), ("bf16", 64)):
        for select in (False, True):
            for hq, hkv in ((8, 2), (32, 8), (1, 1)):
                p = params(hq, hkv, d, kv, sink=4, recent=500, topk=3000)
                for block in (32, 64, 128):
                    last = 0
                    for n in (0, 1, 2, 3, 7, 8, 31, 32, 33, 100, 255, 256, 257, 1000, 2000):
                        row = 0
                        for rows in (1, 31, 32, 33, 100, 1000, 1001, 4095, 4096, 100000, 1 << 20):
                            x = snap.snap_block_decode_workspace(p, n, rows, block, select)
                            assert x >= row and (not select or x >= snap.snap_block_decode_workspace(p, n, rows, block, False))
                            row = x
                        assert row >= last
                        last = row


def test_bad_queries_of_sizes():
    p = params(4, 2, 64)
    for a in ((-1, 100, 32), (1, 0, 32), (1, (1 << 28) + 1, 32), (1, 100, 16), (40000, 100, 32)):
        assert snap.snap_block_decode_workspace(p, *a) == 0
    assert snap.snap_block_decode_workspace(params(34, 2, 64), 1, 100, 32) == 0
    assert snap.snap_block_chosen(params(4, 2, 64, sink=4, recent=65, topk=33), 32) == 1 + 2 + 2
    assert snap.snap_block_chosen(params(4, 2, 64, sink=0, recent=1, topk=0), 128) == 0
    assert snap.snap_block_chosen(p, 48) == 0 and snap.lib().snap_block_chosen(None, 32) == 0


def _pages(call, c, a):
    L, C = snap.lib(), None if c is None else ctypes.byref(c)
    if call == "reserve":
        st = L.snap_pages_reserve(C, a["rows"], a["n"], a["slots"], a["lengths"], a["len"], None, None)
    elif call == "release":
        st = L.snap_pages_release(C, a["rows"], a["n"], a["slots"], None)
    else:
        st = L.snap_pages_map(C, a["rows"], None, a["n"], a["slots"], a["lengths"], a["tokens"], a["starts"], a["seq"], a["row"],
                              a["pos"], None)
    return st, L.snap_last_error().decode()


PAGES = dict(rows=FAKE, n=2, slots=FAKE, lengths=FAKE, len=1, tokens=8, starts=FAKE, seq=FAKE, row=FAKE, pos=FAKE)
P3 = ("reserve", "release", "map")


@pytest.mark.parametrize("calls,c,a,code", [
    (P3, None, {}, INVALID),
    (P3, dict(n_slots=0), {}, INVALID),
    (P3, dict(n_pages=0), {}, INVALID),
    (P3, dict(max_pages=0), {}, INVALID),
    (P3, dict(page_size=8), {}, UNSUPPORTED),
    (P3, dict(page_size=48), {}, UNSUPPORTED),
    (P3, dict(max_pages=(1 << 22) + 1), {}, INVALID),
    (P3, dict(n_pages=1 << 25), {}, UNSUPPORTED),
    (P3, dict(page_table=None), {}, INVALID),
    (("reserve", "release"), dict(held=None), {}, INVALID),
    (("reserve", "release"), dict(free_pages=None), {}, INVALID),
    (("reserve", "release"), dict(n_free=None), {}, INVALID),
    (P3, {}, dict(n=-1), INVALID),
    (P3, {}, dict(n=(1 << 20) + 1), INVALID),
    (P3, {}, dict(rows=None), INVALID),
    (P3, {}, dict(slots=None), INVALID),
    (("reserve",), {}, dict(lengths=None, len=-1), INVALID),
    (("map",), {}, dict(lengths=None), INVALID),
    (("map",), {}, dict(tokens=-1), INVALID),
    (("map",), {}, dict(tokens=(1 << 28) + 1), INVALID),
    (("map",), {}, dict(starts=None), INVALID),
    (("map",), {}, dict(row=None), INVALID),
])
def test_refusals_of_the_page_calls(calls, c, a, code):
    for call in calls:
        st, msg = _pages(call, None if c is None else _pool(**c), {**PAGES, **a})
        assert st == code and msg, (call, st, msg)


@pytest.mark.parametrize("c,a,code", [
    ({}, dict(n=-1), INVALID), ({}, dict(tokens=-1), INVALID), ({}, dict(tokens=(1 << 28) + 1), INVALID),
    (dict(n_pages=1 << 27), {}, UNSUPPORTED), ({}, dict(slots=None), INVALID), ({}, dict(seq=None), INVALID),
    ({}, dict(row=None), INVALID), ({}, dict(pos=None), INVALID), ({}, dict(k=None), INVALID), ({}, dict(v=FAKE + 8), INVALID),
    ({}, dict(ks=(ctypes.c_int64 * 2)(100, 64)), INVALID), (dict(k_scale=None), dict(kv="fp8"), INVALID),
])
def test_refusals_of_the_mapped_append(c, a, code):
    d = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, token=FAKE, weight=FAKE, page_table=FAKE, n_slots=8, n_pages=100,
             page_size=64, max_pages=16)
    b = dict(n=2, slots=FAKE, tokens=8, seq=FAKE, row=FAKE, pos=FAKE, k=FAKE, v=FAKE, ks=None, kv="bf16")
    d.update(c)
    b.update(a)
    L = snap.lib()
    st = L.snap_paged_append_mapped(ctypes.byref(pagedhelp.params(4, 2, 64, b["kv"]).c()), ctypes.byref(snap.SnapPagedCache(**d)), b["n"],
                                    b["slots"], b["tokens"], b["seq"], b["row"], b["pos"], b["k"], b["ks"], b["v"], None, None)
    assert st == code and L.snap_last_error()


def _made():
    p = params(4, 2, 64)
    z = lambda *s, t=torch.int32: torch.zeros(s, dtype=t)  # noqa: E731
    k = z(10, 2, 64, 64, t=torch.int8)
    sc, tail = z(10, 2, 2, t=torch.float32), z(4, 2, 32, 64, t=torch.bfloat16)
    c = snap.block_cache_struct(k, k.clone(), z(4, 8), 32, sc, sc.clone(), tail, tail.clone(), z(10, 2, 2, 2, 64, t=torch.int8), sc.clone())
    new, q = z(2, 2, 1, 64, t=torch.bfloat16), z(2, 4, 64, t=torch.bfloat16)
    pool = snap.page_pool_struct(z(4, 8), z(4), z(10), z(1), 64)
    return dict(p=p, c=c, pool=pool, rows=z(4), ids=z(2), new=new, q=q, out=torch.zeros_like(q), ws=z(1 << 20, t=torch.uint8),
                lengths=z(2), starts=z(3), t=z(5), packed=z(5, 2, 64, t=torch.bfloat16),
                sel=z(2, 2, snap.snap_block_chosen(p, 32)))


CALLS = {
    "append": (lambda a: snap.snap_block_append(a["p"], a["c"], a["rows"], a["ids"], a["new"], a["new"]), ("c", "rows", "ids", "new")),
    "packed": (lambda a: snap.snap_block_append(a["p"], a["c"], a["rows"], a["ids"], a["packed"], a["packed"], starts=a["starts"]),
               ("rows", "packed", "starts")),
    "attn": (lambda a: snap.snap_block_decode_attn(a["p"], a["c"], a["rows"], a["ids"], a["q"], a["out"], a["ws"]),
             ("c", "rows", "ids", "q", "out", "ws")),
    "step": (lambda a: snap.snap_block_decode_step(a["p"], a["c"], a["rows"], a["ids"], a["q"], a["new"], a["new"], a["out"], a["ws"]),
             ("c", "rows", "ids", "q", "new", "out", "ws")),
    "reserve": (lambda a: snap.snap_pages_reserve(a["pool"], a["rows"], a["ids"], a["lengths"]), ("pool", "rows", "ids", "lengths")),
    "release": (lambda a: snap.snap_pages_release(a["pool"], a["rows"], a["ids"]), ("pool", "rows", "ids")),
    "map": (lambda a: snap.snap_pages_map(a["pool"], a["rows"], a["ids"], a["lengths"], a["starts"], a["t"], a["t"], a["t"]),
            ("pool", "rows", "ids", "lengths", "starts", "t")),
}


@pytest.mark.parametrize("call,missing", [(n, m) for n, (_, ms) in CALLS.items() for m in ms])
def test_missing_tensors_are_refused(call, missing):
    with pytest.raises(snap.SnapError):
        CALLS[call][0]({**_made(), missing: None})


def test_tensors_that_do_not_fit_are_refused():
    a = _made()
    p, c = a["p"], a["c"]
    k, table = c.tensors[0], c.tensors[2]
    step = lambda **o: snap.snap_block_decode_step(p, c, *(o.get(x, a[x]) for x in ("rows", "ids", "q", "new", "new", "out", "ws")),  # noqa: E731
                                                   **{x: o[x] for x in ("select", "sel_out") if x in o})
    for bad in (
        lambda: snap.block_cache_struct(k, None, table, 32),
        lambda: snap.block_cache_struct(k, k[:5], table, 32),
        lambda: snap.block_cache_struct(k.float(), k.float(), table, 32),
        lambda: snap.block_cache_struct(k, k, table, 48),
        lambda: snap.block_cache_struct(k, k, table, 128),
        lambda: snap.block_cache_struct(k, k, table.long(), 32),
        lambda: snap.block_cache_struct(k, k, table, 32, k_scale=c.tensors[3][:5]),
        lambda: snap.block_cache_struct(k, k, table, 32, k_tail=c.tensors[5].float()),
        lambda: snap.block_cache_struct(k, k, table, 32, bound=c.tensors[7][..., :32]),
        lambda: snap.page_pool_struct(table, a["rows"]),
        lambda: snap.page_pool_struct(table, a["rows"][:3], a["t"], a["ids"][:1]),
        lambda: snap.page_pool_struct(table, a["rows"], a["t"], a["ids"]),
        lambda: step(q=a["q"].float()), lambda: step(new=a["new"][:, :, :, :32]), lambda: step(out=a["out"].half()),
        lambda: step(rows=a["rows"].long()), lambda: step(rows=a["rows"][:2]), lambda: step(sel_out=a["sel"]),
        lambda: step(select=True, sel_out=a["sel"][..., :-1]),
        lambda: snap.snap_block_append(params(4, 2, 64, "fp8"), c, a["rows"], a["ids"], a["new"], a["new"]),
        lambda: snap.snap_block_append(p, c, a["rows"], a["ids"], a["packed"], a["packed"]),
        lambda: snap.snap_block_append(p, c, a["rows"], a["ids"], a["new"], a["new"], starts=a["starts"]),
        lambda: snap.snap_block_append(p, c, a["rows"], a["ids"], a["packed"], a["packed"], starts=a["starts"], lengths=a["lengths"]),
        lambda: snap.snap_block_append(p, c, a["rows"], a["ids"], a["new"], a["new"], max_len=1),
        lambda: snap.snap_pages_reserve(a["pool"], a["rows"], a["ids"], -1),
        lambda: snap.snap_pages_map(a["pool"], a["rows"], a["ids"], a["lengths"], a["starts"], a["t"], a["t"][:4], a["t"]),
        lambda: snap.snap_pages_map(a["pool"], a["rows"], a["ids"], a["lengths"], a["ids"], a["t"], a["t"], a["t"]),
    ):
        with pytest.raises(snap.SnapError):
            bad()
