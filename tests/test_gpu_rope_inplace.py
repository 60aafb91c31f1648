"""snap_rope with one operand in place and the other not: of the one in place only the rotated dims are touched, so that
its other dims may be where the other operand goes.  Every case prints what names it before touching the GPU."""
import pytest
import torch

import paper_2511_03092_amd as snap

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rot,dtype", [(64, torch.bfloat16), (64, torch.float32), (26, torch.bfloat16)])  # pieces, single dims
@pytest.mark.parametrize("layout", [snap.SNAP_ROPE_HALVES, snap.SNAP_ROPE_PAIRS])
@pytest.mark.parametrize("first", ["q", "k"])
@pytest.mark.parametrize("tokens", [1, 517])
def test_the_other_operand_goes_where_the_one_in_place_is_not_rotated(rot, dtype, layout, first, tokens):
    """Rows of 256: one operand is dims 0 .. 127, in place, of which the first `rot` are rotated; the other's output is
    dims 128 - its width .. 255."""
    print(f"\n[case] rope, {first} in place beside the other's output, rot {rot}, {dtype}, layout {layout}, {tokens} tokens", flush=True)
    g = torch.Generator().manual_seed(3)
    n, heads, d = 2, 3, 128
    wide = torch.randn((n, heads, tokens, 256), generator=g).to(dtype).cuda()
    other = torch.randn((n, heads, tokens, d), generator=g).to(dtype).cuda()
    pos, slots = torch.tensor([100, 7], dtype=torch.int32).cuda(), torch.tensor([1, 0], dtype=torch.int32).cuda()
    r = snap.RopeParams(0, rot, layout=layout)
    # each by itself
    alone, moved = wide[..., :d].contiguous(), torch.empty_like(other)
    snap.snap_rope(r, alone, pos=pos, slot_ids=slots)
    snap.snap_rope(r, other, q_out=moved, pos=pos, slot_ids=slots)
    want = wide.clone()
    want[..., :rot] = alone[..., :rot]
    want[..., rot:rot + d] = moved
    here, there = wide[..., :d], wide[..., rot:rot + d]
    if rot == 26:  # (an output of single dims need not be aligned to pieces)
        assert there.data_ptr() % 16
    if first == "q":
        snap.snap_rope(r, here, other, k_out=there, pos=pos, slot_ids=slots)
    else:
        snap.snap_rope(r, other, here, q_out=there, pos=pos, slot_ids=slots)
    torch.cuda.synchronize()
    assert torch.equal(wide, want)
