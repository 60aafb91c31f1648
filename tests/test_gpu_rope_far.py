"""snap_rope at positions near and past 2^31, against angles formed in whole numbers (200 bits after the point).

Tolerance, by arithmetic (u = 2^-24): the remainder of the angle is rounded to fp32 once, at most pi / 4 (u / 2); the
frequencies and the products before it are off by at most u / 4 at position 2^31.  Sine and cosine are sums whose last
rounding is u / 2, those inside them u / 2 together, what they leave out u / 32.  So each is off by 1.8 u, the product
x2 s by another u / 2 of it: under 3 u (|x1| + |x2|), and half a step of the output."""
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import U

pytestmark = pytest.mark.gpu

BITS = 200


def _turns(base, pairs, factor):
    """Turns a position of every pair, times 2^BITS."""
    getcontext().prec = 90
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211707")
    ln = Decimal(float(np.float32(base))).ln()
    return [int((ln * Decimal(-i) / pairs).exp() / (2 * pi * Decimal(factor)) * 2 ** BITS) for i in range(pairs)]


@pytest.mark.parametrize("base,factor", [(10000.0, 1.0), (500000.0, 1.0), (10000.0, 1.5)])
@pytest.mark.parametrize("layout", [snap.SNAP_ROPE_HALVES, snap.SNAP_ROPE_PAIRS])
@pytest.mark.parametrize("d", [64, 66])  # 16-byte pieces, and pairs by themselves
@pytest.mark.parametrize("start", [(1 << 31) - 3000, 1 << 24, (1 << 30) + 12345])
def test_angles_of_far_positions(base, factor, layout, d, start):
    tokens, pairs = 5000, 32
    rule = snap.SNAP_ROPE_DIVIDE if factor != 1.0 else snap.SNAP_ROPE_PLAIN
    print(f"\n[case] rope at positions from {start}, base {base}, divided by {factor}, layout {layout}, d {d}", flush=True)
    r = snap.RopeParams(0, 64, layout=layout, rule=rule, base=base, factor=factor)
    g = torch.Generator().manual_seed(1)
    x = torch.randn((1, 2, tokens, d), generator=g)
    x[:, 0] = 0  # the first head is (1, 0) in every pair: it turns into (cos, sin)
    one = np.arange(pairs) * (2 if layout == snap.SNAP_ROPE_PAIRS else 1)
    two = one + (1 if layout == snap.SNAP_ROPE_PAIRS else pairs)
    x[:, 0][..., torch.from_numpy(one)] = 1
    q = x.cuda()
    snap.snap_rope(r, q, pos=torch.tensor([start], dtype=torch.int32).cuda(), slot_ids=torch.zeros(1, dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    got, x = q.cpu().double().numpy(), x.double().numpy()
    mask, turns = (1 << BITS) - 1, _turns(base, pairs, factor)
    frac = np.array([[((p * t) & mask) / (1 << BITS) for t in turns] for p in range(start, start + tokens)])
    c, s = np.cos(2 * np.pi * frac), np.sin(2 * np.pi * frac)
    x1, x2 = x[..., one], x[..., two]
    for i, want in ((one, x1 * c - x2 * s), (two, x2 * c + x1 * s)):
        err = np.abs(got[..., i] - want) / U
        tol = 3 * (np.abs(x1) + np.abs(x2)) + np.abs(want)
        over = float((err - tol).max())
        assert over <= 0, (over, float(err[0, 0].max()))
