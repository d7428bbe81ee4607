"""The KL term alone, value and gradient: advantages of 0 and log-probabilities of 0 leave
tok_loss = K = e^x - x - 1 and dlogp = 1 - e^x of x = ref_logp as it is.

Tolerances, u = 2^-24.  |x| < 1: the series' terms in h = x / 2 are of one sign after the first
two, its fused products add 4 u to e^h - 1 - h and its end 2^-28.5 (0.05 u); of e^h - 1 that makes 3 u
(the two cancel by a quarter at most), of its square 7 u; K's two terms are not negative: 9 u of K,
and K + x is 2 u more of |x| + K.  From 1 on: expf is within 2 units of its last place (4 u), and each
difference is rounded: 6 u of e^x + 1 + |x|.  Below the normal numbers (|x| under 1e-19) a rounding is
off by 2^-150 instead: h h, that times the series (about 1/2) and the last sum are one each, so
2 (2^-150 / 2 + 2^-150) + 2^-150 = 2^-148."""
import pytest
import torch

import paper_2608_09703_gb300 as mls

U = 2.0 ** -24


def points():
    x = [torch.linspace(-0.9999999, 0.9999999, 4001), torch.linspace(-0.51, -0.47, 501), torch.linspace(0.47, 0.51, 501)]
    x += [s * torch.logspace(-30, 0, 1500)[:-1] for s in (-1.0, 1.0)]
    x += [torch.linspace(-80.0, -1.0, 500), torch.linspace(1.0, 80.0, 500), torch.tensor([0.0, -0.0, 1.0, -1.0])]
    return torch.cat(x).float()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [4000, 0])
def test_series_and_difference(T):
    x = points()
    x = x[:T] if T else x
    n = len(x)
    ref = x.cuda()[None]
    zero, y = torch.zeros(1, n, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    op = mls.PolicyLoss(n, 10, beta=1.0, agg="sum")
    op(zero, zero, zero[0], y, ref_logp=ref)
    xd = x.double()
    e = torch.exp(xd)
    # K in 64 bits without the difference: its own series where that is short
    K = torch.where(xd.abs() < 0.05, sum(xd ** k / float(torch.lgamma(torch.tensor(k + 1.0, dtype=torch.float64)).exp())
                                         for k in range(2, 14)), torch.expm1(xd) - xd)
    near = xd.abs() < 1
    tol = torch.where(near, 9 * U * K, 6 * U * (e + 1 + xd.abs())) + 2.0 ** -148
    got = op.tok_loss[0].cpu().double()
    assert bool((got >= 0).all())
    bad = ~((got - K).abs() <= tol)
    assert not bad.any(), (x[bad][:5], ((got - K).abs() / tol)[bad][:5])
    g, want = op.dlogp[0].cpu().double(), -torch.expm1(xd)
    tolg = torch.where(near, 2 * U * (xd.abs() + K) + 9 * U * K, 6 * U * (e + 1)) + 2.0 ** -148
    bad = ~((g - want).abs() <= tolg)
    assert not bad.any(), (x[bad][:5], ((g - want).abs() / tolg)[bad][:5])
