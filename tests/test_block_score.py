"""The score that selects blocks, from its definition, against the products it stands for (CPU)."""
from types import SimpleNamespace

import pytest
import torch

from blockhelp import scale_of, scores


@pytest.mark.parametrize("d,block", [(64, 32), (128, 64)])
def test_products_exceed_the_score_by_the_query_s_rounding_at_most(d, block):
    """u / 2 sum |k| a query, and roundings of fp32: u = 2^-24 for each of d terms of the products here (float64 otherwise),
    and for the quotients, the scales and the three products of the score."""
    g = torch.Generator().manual_seed(1)
    n = 40
    k = (torch.randn((n * block, 1, d), generator=g) * (0.1 + torch.rand(d, generator=g))).bfloat16()
    q = torch.randn((4, d), generator=g).bfloat16()
    for j in range(n):  # some blocks of rows that are alike, of a query's signs
        if j % 2:
            k[j * block:(j + 1) * block, 0] = (torch.sign(q[j % 4].float()) * k[j * block:(j + 1) * block, 0].float().abs().amax(0)).bfloat16()
    c = SimpleNamespace(x={"k": [k]}, block=block)
    s = scores(c, 0, 0, q, range(n))
    f = q.double()
    unit = scale_of(q.float()[:, None], 127.0).double()
    for j in range(n):
        x = k[j * block:(j + 1) * block, 0].double()
        products = f @ x.T
        slack = unit[:, None] / 2 * x.abs().sum(1) + 8 * 2.0 ** -24 * (f.abs() @ x.abs().T)
        assert (products <= float(s[j]) + slack).all(), j


def test_a_product_can_exceed_the_score():
    """A query whose small dims round to no code: each is 0.0037, below half of u = 1 / 127, and all of them count in q.k."""
    d, block = 64, 32
    q = torch.full((1, d), 0.0037).bfloat16()
    q[0, 0] = 1.0
    k = torch.ones((block, 1, d), dtype=torch.bfloat16)
    s = scores(SimpleNamespace(x={"k": [k]}, block=block), 0, 0, q, [0])
    assert abs(float(s[0]) - 1.0) < 1e-5 and float(q.double().sum()) > 1.2
