"""snap_paged_append of inputs whose strides along sizes of one say nothing.  Every case prints what names it before
touching the GPU."""
import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import Paged
from test_gpu_paged import _i32, _shape

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,heads,tokens", [(1, 2, 5), (3, 1, 5), (3, 2, 1), (1, 1, 1)])
def test_strides_along_sizes_of_one_are_ignored(n, heads, tokens):
    """A view's stride along a size of one may be anything, odd and 0 among it."""
    p, kv, page = _shape("d64-fp8", n_kv_heads=heads)
    print(f"\n[case] paged append, {n} sequences x {heads} heads x {tokens} tokens, strides of 3 along sizes of one", flush=True)
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn((n, heads, tokens, 64), generator=g).bfloat16().cuda() for _ in range(2))
    state = []
    for odd in (False, True):
        c = Paged(p, kv, n, page, [tokens] * n, 1)
        if odd:
            k, v = (x.as_strided(x.shape, [3 if s == 1 else st for s, st in zip(x.shape[:3], x.stride())] + [1]) for x in (k, v))
        snap.snap_paged_append(p, c.c, c.rows, c.pos, _i32(list(range(n))), k, v)
        torch.cuda.synchronize()
        state.append(c.state())
    for x in ("k", "v", "token", "weight"):
        assert torch.equal(state[0][x].view(torch.uint8), state[1][x].view(torch.uint8)), x


def test_odd_strides_along_larger_sizes_are_refused():
    p, kv, page = _shape("d64-fp8")
    print("\n[case] paged append, a head stride of 68 elements", flush=True)
    c = Paged(p, kv, 1, page, [1], 1)
    k = torch.zeros((1, 2, 1, 68), dtype=torch.bfloat16, device="cuda")[..., :64]
    with pytest.raises(snap.SnapError) as e:
        snap.snap_paged_append(p, c.c, c.rows, c.pos, _i32([0]), k, k)
    assert e.value.status == snap.SNAP_ERR_INVALID_ARG
