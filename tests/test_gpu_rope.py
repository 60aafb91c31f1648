"""snap_rope against the rotation in float64: layouts, part of a head, the frequency rules, types, strides, in place,
ragged lengths, far positions, skipped slots.  Every case prints what names it before touching the GPU."""
import numpy as np
import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import HALF_STEP, U, rope

pytestmark = pytest.mark.gpu

R = snap.RopeParams
CASES = {
    # params, dtype, n, heads of q and k, tokens, d, first position at most
    "halves-step": (R(0, 128, base=500000.0), "bf16", 5, (32, 8), 1, 128, 131072),
    "halves-prompt": (R(0, 128, base=500000.0), "bf16", 2, (4, 2), 333, 128, 1),
    "pairs-step": (R(0, 64, layout=snap.SNAP_ROPE_PAIRS), "bf16", 3, (8, 8), 1, 64, 5000),
    "pairs-f32": (R(0, 64, layout=snap.SNAP_ROPE_PAIRS), "f32", 2, (4, 2), 65, 64, 1 << 20),
    "halves-f32-far": (R(0, 64), "f32", 3, (4, 2), 3, 64, (1 << 31) - 10),
    "part-front": (R(0, 32), "bf16", 2, (4, 1), 17, 64, 100),
    "part-back-latent": (R(512, 64, layout=snap.SNAP_ROPE_PAIRS), "bf16", 2, (8, 1), 19, 576, 9000),
    "odd-part-halves": (R(3, 10), "bf16", 2, (3, 1), 7, 40, 100),
    "odd-part-pairs-f32": (R(1, 6, layout=snap.SNAP_ROPE_PAIRS), "f32", 2, (3, 1), 7, 9, 100),
    "two-dims": (R(0, 2), "f32", 1, (1, 0), 5, 2, 100),
    "divide": (R(0, 128, rule=snap.SNAP_ROPE_DIVIDE, factor=4.0), "bf16", 2, (4, 2), 9, 128, 100000),
    "turns": (R(0, 128, rule=snap.SNAP_ROPE_BY_TURNS, base=500000.0, factor=8.0, high_turns=4.0, orig_len=8192), "f32",
              2, (4, 2), 9, 128, 131072),
    "index": (R(0, 64, rule=snap.SNAP_ROPE_BY_INDEX, factor=40.0, orig_len=4096, amplitude=1.25,
                layout=snap.SNAP_ROPE_PAIRS), "f32", 2, (4, 2), 9, 64, 131072),
    "long-prompt": (R(0, 64), "bf16", 1, (2, 1), 20011, 64, 1),
}


def _make(name, packed=False):
    r, dt, n, (hq, hk), tokens, d, far = CASES[name]
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[dt]
    g = torch.Generator().manual_seed(len(name) + 3 * tokens)
    if packed:  # token by token, the heads of q, k and v side by side
        x = torch.randn((n, tokens, hq + 2 * hk, d), generator=g).to(dtype).cuda()
        q, k = x[:, :, :hq].transpose(1, 2), x[:, :, hq:hq + hk].transpose(1, 2)
    else:
        q = torch.randn((n, hq, tokens, d), generator=g).to(dtype).cuda()
        k = torch.randn((n, hk, tokens, d), generator=g).to(dtype).cuda()
    pos = torch.randint(0, far, (n + 2,), generator=g, dtype=torch.int32)
    slots = torch.randperm(n + 2, generator=g)[:n].to(torch.int32)
    return r, q, k if hk else None, pos, slots


def _check(r, before, after, first, lengths, untouched=None):
    x = before.double().cpu().numpy()
    at = np.asarray(first, np.float64)[:, None, None] + np.arange(x.shape[2])[None, None, :]
    want, size = rope(r, x, np.broadcast_to(at, x.shape[:3]))
    tol = HALF_STEP[after.dtype] * np.abs(want) * (1 + 2.0 ** -8) + 8 * U * size
    err = np.abs(after.double().cpu().numpy() - want)
    for b, n in enumerate(lengths):
        assert (err[b, :, :n] <= tol[b, :, :n]).all(), (b, float((err[b, :, :n] - tol[b, :, :n]).max()))
        if untouched is not None:
            assert torch.equal(after[b, :, n:], untouched[b, :, n:])


@pytest.mark.parametrize("name", list(CASES))
def test_rope_of_its_own_buffers(name):
    r, q, k, pos, slots = _make(name)
    print(f"\n[case] rope {name}", flush=True)
    yq, yk = torch.full_like(q, 5.0), None if k is None else torch.full_like(k, 5.0)
    first = pos[slots.long()].numpy()
    snap.snap_rope(r, q, k, yq, yk, pos=pos.cuda(), slot_ids=slots.cuda())
    torch.cuda.synchronize()
    full = [q.shape[2]] * q.shape[0]
    _check(r, q, yq, first, full)
    if k is not None:
        _check(r, k, yk, first, full)


@pytest.mark.parametrize("name", ["halves-prompt", "pairs-f32", "part-back-latent", "odd-part-halves", "turns"])
def test_rope_in_place_ragged_and_from_position_zero(name):
    """In place, only live tokens and rotated dims change; without pos a token is at its index; the result is that of
    the call into other buffers."""
    r, q, k, pos, slots = _make(name)
    n, _, tokens, _ = q.shape
    lengths = [tokens // 2, tokens + 5, 0, 1][:n]
    live = [min(x, tokens) for x in lengths]
    print(f"\n[case] rope in place {name}: lengths {lengths}", flush=True)
    q0, k0, lt = q.clone(), k.clone(), torch.tensor(lengths, dtype=torch.int32).cuda()
    yq, yk = torch.full_like(q, 5.0), torch.full_like(k, 5.0)
    snap.snap_rope(r, q, k, yq, yk, lengths=lt)
    snap.snap_rope(r, q, k, lengths=lt)
    torch.cuda.synchronize()
    _check(r, q0, q, [0] * n, live, untouched=q0)
    _check(r, k0, k, [0] * n, live, untouched=k0)
    _check(r, q0, yq, [0] * n, live, untouched=torch.full_like(q, 5.0))
    for b, m in enumerate(live):
        assert torch.equal(q[b, :, :m], yq[b, :, :m]) and torch.equal(k[b, :, :m], yk[b, :, :m])


@pytest.mark.parametrize("name", ["halves-prompt", "halves-step", "part-back-latent", "odd-part-pairs-f32", "index"])
def test_rope_of_a_packed_projection(name):
    """q and k as views of one token-by-token buffer: into head-by-head buffers and into slices of wider rows, the
    other elements of which stay."""
    r, q, k, pos, slots = _make(name, packed=True)
    print(f"\n[case] rope packed {name}", flush=True)
    n, hq, tokens, d = q.shape
    wide = torch.full((n, hq, tokens, d + 24), 5.0, dtype=q.dtype, device="cuda")
    yk = torch.empty(k.shape, dtype=k.dtype, device="cuda")
    first = pos[slots.long()].numpy()
    snap.snap_rope(r, q, k, wide[..., 8:8 + d], yk, pos=pos.cuda(), slot_ids=slots.cuda())
    torch.cuda.synchronize()
    _check(r, q, wide[..., 8:8 + d], first, [tokens] * n)
    _check(r, k, yk, first, [tokens] * n)
    assert bool((wide[..., :8] == 5.0).all()) and bool((wide[..., 8 + d:] == 5.0).all())


def test_rope_skips_slots_that_are_not_there_and_repeats_a_broadcast_input():
    r = R(0, 64)
    print("\n[case] rope: slots -1 and 9 of 4, x broadcast over the heads", flush=True)
    x = torch.randn((3, 1, 5, 64), device="cuda").expand(3, 4, 5, 64)
    y = torch.full((3, 4, 5, 64), 7.0, device="cuda")
    pos = torch.tensor([3, 2, 1, 0], dtype=torch.int32).cuda()
    snap.snap_rope(r, x, q_out=y, pos=pos, slot_ids=torch.tensor([-1, 1, 9], dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert bool((y[0] == 7.0).all()) and bool((y[2] == 7.0).all())
    _check(r, x[1:2], y[1:2], [2], [5])


def test_rope_replays_in_a_graph():
    r, q, k, pos, slots = _make("halves-step")
    print("\n[case] rope captured and replayed at later positions", flush=True)
    yq, yk, p, s = torch.empty_like(q), torch.empty_like(k), pos.cuda(), slots.cuda()
    snap.snap_rope(r, q, k, yq, yk, pos=p, slot_ids=s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        snap.snap_rope(r, q, k, yq, yk, pos=p, slot_ids=s)
        snap.snap_advance(p, s)
    for step in range(3):
        first = p[s.long()].cpu().numpy()
        graph.replay()
        torch.cuda.synchronize()
        _check(r, q, yq, first, [1] * 5)
        _check(r, k, yk, first, [1] * 5)
        assert torch.equal(p[s.long()].cpu(), torch.from_numpy(first) + 1)
