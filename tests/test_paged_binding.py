"""Tensors that are missing: the binding raises SnapError, as for those that do not fit (no GPU)."""
import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import params


def _made():
    p = params(8, 2, 64)
    k = torch.zeros((10, 2, 16, 64), dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    c = snap.paged_cache_struct(k, k.clone(), i32(4, 8), i32(10, 2, 16), torch.zeros((10, 2, 16)))
    new, q = torch.zeros((2, 2, 1, 64), dtype=torch.bfloat16), torch.zeros((2, 8, 64), dtype=torch.bfloat16)
    return dict(p=p, c=c, rows=i32(4), pos=i32(4), ids=i32(2), new=new, q=q, out=torch.zeros_like(q),
                ws=torch.zeros(1 << 20, dtype=torch.uint8), rows_out=i32(4))


CALLS = {
    "append": (lambda a: snap.snap_paged_append(a["p"], a["c"], a["rows"], a["pos"], a["ids"], a["new"], a["new"]),
               ("c", "rows", "ids", "new")),
    "attn": (lambda a: snap.snap_paged_decode_attn(a["p"], a["c"], a["rows"], a["ids"], a["q"], a["out"], a["ws"]),
             ("c", "rows", "ids", "q", "out", "ws")),
    "step": (lambda a: snap.snap_paged_decode_step(a["p"], a["c"], a["rows"], a["pos"], a["ids"], a["q"], a["new"], a["new"],
                                                   a["out"], a["ws"]), ("c", "rows", "ids", "q", "new", "out", "ws")),
    "evict": (lambda a: snap.snap_paged_evict(a["p"], a["c"], a["rows"], a["pos"], a["ids"], a["rows_out"], a["ws"]),
              ("c", "rows", "pos", "ids", "rows_out", "ws")),
    "rope": (lambda a: snap.snap_rope(snap.RopeParams(0, 64), a["new"], pos=a["pos"], slot_ids=a["ids"]), ("new", "ids")),
}


@pytest.mark.parametrize("call,missing", [(n, m) for n, (_, ms) in CALLS.items() for m in ms])
def test_missing_tensors_are_refused(call, missing):
    with pytest.raises(snap.SnapError):
        CALLS[call][0]({**_made(), missing: None})


def test_a_cache_without_keys_or_table_is_refused():
    k, table = torch.zeros((10, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((4, 8), dtype=torch.int32)
    for bad in (lambda: snap.paged_cache_struct(None, k, table), lambda: snap.paged_cache_struct(k, k, None)):
        with pytest.raises(snap.SnapError):
            bad()


@pytest.mark.gpu
@pytest.mark.parametrize("call", ["attn", "step", "evict"])
def test_a_missing_workspace_is_the_librarys_to_refuse(call):
    """Its status, and none where no sequence is there."""
    print(f"\n[case] paged {call} without a workspace", flush=True)
    a = {x: v.cuda() if isinstance(v, torch.Tensor) else v for x, v in _made().items()}
    k = torch.zeros((10, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    a.update(c=snap.paged_cache_struct(k, k.clone(), i32(4, 8), i32(10, 2, 16), torch.zeros((10, 2, 16), device="cuda")), ws=None)
    with pytest.raises(snap.SnapError) as e:
        CALLS[call][0](a)
    assert e.value.status == snap.SNAP_ERR_WORKSPACE
    CALLS[call][0]({**a, "ids": a["ids"][:0], "q": a["q"][:0], "new": a["new"][:0], "out": a["out"][:0]})
    torch.cuda.synchronize()
