"""What attention over the paged cache computes with 32 bits: probabilities of 16-bit and fp8 rows enter the value
product whole (latent rows: 2^-18 off at most), so that an fp32 output is about as exact as the sums are.  Every case
prints what names it before touching the GPU.

Tolerances, by arithmetic (u = 2^-24, a rounding to fp32 is off by at most u relative).  Where every value is the same
the output is that value, whatever the probabilities: the same ones are in the product and in the sum below it.  What is
left are the roundings of the two sums, whose terms have one sign: u for each addition on a term's way (an item's blocks,
the 32 rows of one, lanes, waves or items), and 8 u for the references' exp2, the reciprocal and the products."""
import math

import pytest
import torch

import paper_2511_03092_amd as snap
from pagedhelp import U, Paged, fill
from test_gpu_paged import SHAPES, _shape

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", [x for x in SHAPES if SHAPES[x][4] != "f32"])
@pytest.mark.parametrize("length", [300, 3000])
def test_probabilities_lose_no_bits_before_the_values(name, length):
    """Values that are all one, so that their weighted mean is: the first row of every 32 has logit 0, the others the one
    whose exp is half of 1 + 2^-7 - 2^-17, which two terms of 8 bits, cut off, would miss by 2^-15 - 2^-17, 384 u."""
    p, kv, page = _shape(name)
    print(f"\n[case] paged decode {name} of {length} rows, values all one", flush=True)
    c = fill(Paged(p, kv, 1, page, [length], 1), [0], [length], 2)
    one = {"bf16": 1.0, "fp8": 0x38}[kv]
    at = p.d_qk - 3  # three dims tell the rows apart; the queries are zero in the others
    c.k[:], c.k[..., at:] = one, one
    if c.v is not None:
        c.v[:] = one
    for pg, off in c.places(0, length)[::32]:
        c.k[pg, :, off, at:] = 0
    G = p.n_q_heads // p.n_kv_heads
    q = torch.zeros((1, p.n_q_heads, p.d_qk), dtype=torch.bfloat16)
    scale = torch.ones(p.n_kv_heads) if kv == "bf16" else c.k_scale[0].cpu()
    for h in range(p.n_q_heads):
        rest = math.log(0.5 * (1 + 2.0 ** -7 - 2.0 ** -17)) * math.sqrt(p.d_qk) / float(scale[h // G])
        for i in range(3):  # to 24 bits
            q[0, h, at + i] = rest
            rest -= float(q[0, h, at + i])
    c.rows[0] = length - 1
    out = torch.empty((1, p.n_q_heads, p.d_v), dtype=torch.float32, device="cuda")
    ws = snap.workspace(snap.snap_paged_decode_workspace(p, 1, length, False))
    snap.snap_paged_decode_attn(p, c.c, c.rows, torch.zeros(1, dtype=torch.int32, device="cuda"), q.cuda(), out, ws,
                                max_rows=length)
    torch.cuda.synchronize()
    want = torch.ones((1, p.n_q_heads, 1), dtype=torch.float64)
    if kv == "fp8":
        want *= (c.k_scale if p.v_in_k else c.v_scale)[0].double().cpu().repeat_interleave(G)[None, :, None]
    cols = at if p.d_v == p.d_qk and p.v_in_k else p.d_v  # (dims that hold the same value in every row)
    # an item has all blocks at most: length / 32 + 32 + 5 additions on a term's way, twice
    tol = (2 * (length / 32 + 37) + 8) * U + (2.0 ** -18 if p.d_qk == 576 else 0.0)
    err = float(((out.double().cpu() - want).abs() / want)[..., :cols].max())
    assert err <= tol, (err / U, tol / U)
