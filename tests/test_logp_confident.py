"""Tokens that have nearly all of the mass, as most of a model's own samples do.  A row of H is
one unit vector, so the logits are the heads' bf16 values without an error, and what is left is
the arithmetic of the softmax.

Tolerances, u = 2^-24, with x = (z - m) log2(e) / tau for the largest logit m.  z - m is rounded,
log2(e) / tau is rounded, and so is their product: 3 u |x| in the exponent, as much (times ln 2) of
the term.  The hardware's 2^x adds 4 u (2^-22), each change of the running maximum 8 u (its factor
and two products), the sums 32 u; the largest logit's own term is 1.  Its columns, the 8 sums of 16
of a tile's 128, are added to that 1: there an addition is off by at most u, and by no more than what is
added, which the next words never see again: 24 u, or twice those columns' terms if that is less.
"""
import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B

U = 2.0 ** -24
D = 64


def inputs(T, V, scale, gap, alone=False, seed=0, models=1):
    """T tokens over the D unit vectors; token t's target has logit `scale`, the others spread
    around scale - gap; `alone`: none of any size in the target's 128 columns."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = torch.arange(T, device="cuda") % D
    H = [torch.eye(D, device="cuda").bfloat16()[k] for _ in range(models)]
    best = torch.randint(0, V, (D,), generator=g, device="cuda")
    W = []
    for _ in range(models):
        w = (2.5 * torch.randn(V, D, generator=g, device="cuda")).clamp(max=gap - 1.0) + scale - gap
        if alone:
            near = torch.arange(V, device="cuda")[:, None] // 128 == best // 128
            w = torch.where(near, scale - 200.0, w)
        w[best, torch.arange(D, device="cuda")] = scale
        W.append(w.bfloat16())
    return H, W, best[k].int(), k


def shares(W, y, k, tau, V):
    """Per unit vector and model: what the other tokens add to the target's 1, and how far off."""
    tau = float(torch.tensor(tau))
    z = W.double().t()  # [D, V]
    best = torch.zeros(D, dtype=torch.int64, device="cuda")
    best[k] = y.long()
    x = (z - z.gather(1, best[:, None])) / tau
    e = torch.exp(x).scatter(1, best[:, None], 0.0)
    others = e.sum(1)
    near = (e * (torch.arange(V, device="cuda") // 128 == best[:, None] // 128)).sum(1)
    changes = -(-V // 256) + 16
    tol = U * (e * (3 * x.abs() + 4 + 32 + 8 * changes)).sum(1) + torch.clamp(2 * near, max=24 * U)
    return others[k], tol[k]


CASES = [(64, 5000, 12.0, 20.0, 1.0), (64, 5000, 29.75, 27.0, 1.0), (200, 50304, 41.5, 24.0, 1.0),
         (64, 300, 30.25, 14.0, 0.7), (40, 20000, 100.5, 34.0, 1.0), (20000, 5003, 23.25, 22.0, 1.0),
         (1000, 9000, -57.5, 26.0, 1.3), (64, 2000, 99.0, 60.0, 3.0)]


@pytest.mark.gpu
@pytest.mark.parametrize("alone", [False, True])
@pytest.mark.parametrize("T,V,scale,gap,tau", CASES)
def test_log_probabilities(T, V, scale, gap, tau, alone):
    H, W, y, k = inputs(T, V, scale, gap, alone, seed=V, models=2)
    op = mls.HeadLogp((D, D), T, V, tau=tau)
    logp = op.forward(H, W, y)
    assert bool((logp <= 0).all())
    for m in range(2):
        others, tol = shares(W[m], y, k, tau, V)
        want = -torch.log1p(others)
        err = (logp[m].double() - want).abs()
        bad = ~(err <= tol / (1 + others) + 6 * U * want.abs())
        assert not bad.any(), (int(bad.sum()), float(err.max()), float(others.median()))
    assert mls.mls_get_status() == 0
