"""Layer norm of rows wider than a block caches, and long columns of theirs: sums whose error does
not grow with the width or with the number of rows.

Tolerances, u = 2^-24: a lane adds at most 32 values in fp32 and those in two words, or keeps at most
8 vectors; with the squares, the butterfly, the products with 1 / d and eps a row sum is within
K = 64 u of the sum of its terms' sizes at every width.  The column sums add 8 rows in fp32, those in
two words, and then the blocks' shares, at most 152 (a warp adds ten in a chain, sixteen warps' follow).
"""
import pytest
import torch

import paper_2608_09703_gb300 as mls

U = 2.0 ** -24
K = 64 * U


def alternating(T, d, dtype):
    """Rows of +-a, a different one each: all squares alike, so that a long sum errs to one side."""
    a = 1.1 * (1 + torch.arange(T, device="cuda") % 5)[:, None]
    sign = torch.where(torch.arange(d, device="cuda") % 2 == 0, 1.0, -1.0)
    return (a * sign).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [4104, 16384, 16392, 32768, 32776, 40000, 1 << 20, (1 << 22) + 8, 1 << 24])
def test_row_sums_of_any_width(d, dtype):
    T = 3
    x = alternating(T, d, dtype)
    x[1] += 3.0  # a mean beside the spread
    dy = (0.1 + 0.07 * x.float()).to(dtype)
    op = mls.LayerNorm(T, d, gain=False, bias=False, dtype=dtype)
    op.forward(x)
    op.backward(x, dy)
    ut = torch.finfo(dtype).eps / 2
    for t in range(T):
        xd, gd = x[t].double(), dy[t].double()
        mu = xd.mean()
        r = 1 / ((xd - mu).square().mean() + op.eps).sqrt()
        xh = (xd - mu) * r
        size = xd.abs().mean()
        assert float((op.mean[t].double() - mu).abs()) <= float(K * size)
        assert float((op.rstd[t].double() - r).abs()) <= float(K * r * (1 + (K * size * r) ** 2))
        w = xh.abs() + 1 + r * size
        assert bool(((op.y[t].double() - xh).abs() <= ut * xh.abs() + K * w).all())
        a1, a2 = gd.mean(), (gd * xh).mean()
        dx = r * (gd - a1 - xh * a2)
        bound = ut * dx.abs() + 2 * K * r * (gd.abs() + gd.abs().mean() + w * (gd.abs() * w).mean())
        assert bool(((op.dx[t].double() - dx).abs() <= bound).all())


@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype", [(16392, torch.float32), (32776, torch.bfloat16)])
def test_long_columns(d, dtype):
    """60000 rows of the same gradient: what an fp32 chain of them loses is seen at once."""
    T = 60000
    x = alternating(1, d, dtype).expand(T, d).contiguous()
    dy = torch.full((T, d), 0.1003, device="cuda", dtype=dtype)
    gain = torch.ones(d, device="cuda", dtype=dtype)
    op = mls.LayerNorm(T, d, dtype=dtype)
    op.forward(x, gain, gain)
    op.backward(x, dy, gain)
    g = float(dy[0, 0])
    xd = x[0].double()
    xh = (xd - xd.mean()) / ((xd - xd.mean()).square().mean() + op.eps).sqrt()
    for got, want in ((op.dbias, torch.full((d,), T * g, device="cuda", dtype=torch.float64)), (op.dgain, T * g * xh)):
        assert float(((got.double() - want).abs() / want.abs()).max()) <= (8 + 10 + 16 + 64) * U


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,dtype", [(40, 32776, torch.bfloat16), (33, 40000, torch.bfloat16), (21, 16392, torch.float32),
                                       (300, 65544, torch.bfloat16), (5, 1 << 20, torch.float32)])
def test_in_place(T, d, dtype):
    """y in x's place and dx in dy's, with the column sums of dy taken before it is written over."""
    g = torch.Generator(device="cuda").manual_seed(d)
    x, dy = [torch.randn(T, d, generator=g, device="cuda").to(dtype) for _ in range(2)]
    gain, bias = [torch.randn(d, generator=g, device="cuda").to(dtype) for _ in range(2)]
    op = mls.LayerNorm(T, d, dtype=dtype)
    op.forward(x, gain, bias)
    op.backward(x, dy, gain)
    x2, dy2 = x.clone(), dy.clone()
    mls.mls_layer_norm_fwd(x2, gain, bias, op.eps, x2)
    dg, db = torch.empty_like(op.dgain), torch.empty_like(op.dbias)
    mls.mls_layer_norm_bwd(x, gain, dy2, op.mean, op.rstd, dy2, dg, db, op.ws)
    assert torch.equal(x2, op.y) and torch.equal(dy2, op.dx)
    assert torch.equal(dg, op.dgain) and torch.equal(db, op.dbias)
