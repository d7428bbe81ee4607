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
import ctypes

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from paper_2608_09703_gb300 import build as mbuild

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


def grads(op, H, W, y, scale, plain=False):
    """dL/dz [M][T, V] for dlogp = scale: with T different unit vectors dW is its transpose."""
    T = len(y)
    dl = torch.full((len(H), T), scale, device="cuda")
    if plain:
        B.mls_head_logp_bwd(op.prob, H, W, y, op.lse, dl, op.dH, op.dW, op.ws)
    else:
        op.backward(H, W, y, dl)
    return [w.double().t() for w in op.dW]


@pytest.mark.gpu
@pytest.mark.parametrize("alone", [False, True])
@pytest.mark.parametrize("V,scale,gap,tau,group", [(5000, 12.0, 20.0, 1.0, 0), (5000, 29.75, 27.0, 1.0, 1024),
                                                   (50304, 41.5, 24.0, 1.0, 0), (300, 30.25, 14.0, 0.7, 0),
                                                   (20000, 100.5, 34.0, 1.0, 0), (9000, -57.5, 26.0, 1.3, 2048)])
def test_gradient_at_the_target_and_elsewhere(V, scale, gap, tau, group, alone):
    """1 - p of the target to its own digits (rounded to bf16 in dL/dz, dW is of one token's), the
    other tokens' p within the rounding of lse's one word, 2 u |lse|, and of the exponent, and bf16."""
    H, W, y, k = inputs(D, V, scale, gap, alone, seed=V + 1, models=2)
    op = mls.HeadLogp((D, D), D, V, tau=tau, vocab_group=group)
    op.forward(H, W, y)
    t32 = float(torch.tensor(tau))
    for m, G in enumerate(grads(op, H, W, y, 3.0)):
        others, tol = shares(W[m], y, k, tau, V)
        c = 3.0 / t32
        want = c * others / (1 + others)
        got = G.gather(1, y.long()[:, None])[:, 0]
        assert bool(((got - want).abs() <= c * tol + (2.0 ** -8 + 8 * U) * want).all()), \
            float(((got - want).abs() / want).max())
        z = W[m].double().t() / t32
        p = torch.softmax(z, 1)
        lse = torch.logsumexp(z, 1, keepdim=True)
        off = U * (4 * lse.abs() + 4 * z.abs() + 64) + (tol / (1 + others))[:, None]
        err = (G + c * p).scatter(1, y.long()[:, None], 0.0).abs()
        assert bool((err <= c * p * (off + 2.0 ** -8) + 1e-37).all())
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
def test_other_targets_in_the_backward():
    """Targets that are not the forward's: their own gradients, 1 - p within the rounding of lse."""
    V, scale = 3000, 30.0
    H, W, y, k = inputs(D, V, scale, 22.0, seed=5)
    op = mls.HeadLogp((D,), D, V)
    other = torch.where(torch.arange(D, device="cuda") % 2 == 0, (y + 1) % V, -1).int()
    z = W[0].double().t()
    for first, then in ((other, y), (y, other)):
        op.forward(H, W, first)
        G = grads(op, H, W, then, 1.0)[0]
        on = then >= 0
        at = then.clamp(min=0).long()[:, None]
        p = torch.softmax(z, 1).gather(1, at)[:, 0]
        want, got = 1 - p, G.gather(1, at)[:, 0]
        bound = 4 * U * scale + 64 * U + 2.0 ** -8 * got.abs()
        assert bool(((got - want).abs() <= bound)[on].all()) and not G[~on].any()


@pytest.mark.gpu
def test_without_what_the_forward_hands_on():
    """The plain calls: 1 - p within the rounding of lse."""
    V, scale = 5000, 29.75
    H, W, y, k = inputs(D, V, scale, 27.0, seed=2)
    op = mls.HeadLogp((D,), D, V)
    B.mls_head_logp_fwd(op.prob, H, W, y, op.logp, op.lse, op.ws)
    got = grads(op, H, W, y, 1.0, plain=True)[0].gather(1, y.long()[:, None])[:, 0]
    others, tol = shares(W[0], y, k, 1.0, V)
    want = others / (1 + others)
    assert bool(((got - want).abs() <= tol + 2 * U * scale + 16 * U + 2.0 ** -8 * got.abs()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("d,V,tau", [(136, 20000, 1.0), (520, 1031, 0.8), (2048, 33000, 1.0)])
def test_recomputed_logits_are_the_same(d, V, tau):
    """Any hidden state: one token's dW is dL/dz times its row, so dL/dz at the target is read off dW
    and is 1 - exp of the forward's log-probability, whatever that is."""
    for seed in range(4):
        g = torch.Generator(device="cuda").manual_seed(seed)
        H = [torch.randn(1, d, generator=g, device="cuda").bfloat16()]
        W = [(torch.randn(V, d, generator=g, device="cuda") * (4.0 / d ** 0.5)).bfloat16()]
        best = int((H[0].float() @ W[0].float().t()).argmax())
        W[0][best] = (H[0][0].float() * (24.0 + 2 * seed) / float((H[0].float() ** 2).sum())).bfloat16()
        y = torch.tensor([best], dtype=torch.int32, device="cuda")
        op = mls.HeadLogp((d,), 1, V, tau=tau)
        logp = float(op.forward(H, W, y))
        op.backward(H, W, y, torch.ones(1, 1, device="cuda"))
        h = H[0][0].double()
        got = float((op.dW[0][best].double() * h).sum() / (h * h).sum()) * float(torch.tensor(tau))
        want = -torch.expm1(torch.tensor(logp, dtype=torch.float64)).item()
        assert 0 < want < 0.9 and abs(got - want) <= 2 * 2.0 ** -8 * want, (got, want)


# ------------------------------------------------------------------ refusals
def test_refusals_of_the_library():
    mbuild.build()
    L, prob, p = B.lib(), mls.Problem((64,), 10, 100), 0x1000

    def arr(v):
        return (ctypes.c_void_p * 1)(v)

    def fwd(peak, prob=prob):
        return L.mls_head_logp_fwd_peak(prob.ref(), arr(p), arr(p), p, p, p, peak, 0x10000, 1 << 40, None)

    def bwd(peak, prob=prob):
        return L.mls_head_logp_bwd_peak(prob.ref(), arr(p), arr(p), p, p, peak, p, arr(2 * p), arr(3 * p), 0x10000,
                                        1 << 40, None)

    for call in (fwd, bwd):
        assert call(None) == B.MLS_ERR_ARG and call(p + 2) == B.MLS_ERR_ALIGN
        assert call(p, mls.Problem((64,), 10, 100, in_dtype=B.MLS_FP32)) == B.MLS_ERR_UNSUPPORTED
    assert L.mls_head_logp_fwd_peak(*[None] * 8, 0, None) == B.MLS_ERR_ARG
    assert L.mls_head_logp_bwd_peak(*[None] * 10, 0, None) == B.MLS_ERR_ARG


@pytest.mark.gpu
def test_refusals_of_the_binding():
    H, W, y, _ = inputs(D, 500, 10.0, 12.0)
    op = mls.HeadLogp((D,), D, 500)
    dl = torch.ones(1, D, device="cuda")
    for peak in (op.peak[0], op.peak.double(), op.peak.cpu(), op.peak.transpose(0, 1)[:, :, 1:]):
        with pytest.raises((TypeError, ValueError)):
            B.mls_head_logp_fwd(op.prob, H, W, y, op.logp, op.lse, op.ws, peak=peak)
        with pytest.raises((TypeError, ValueError)):
            B.mls_head_logp_bwd(op.prob, H, W, y, op.lse, dl, op.dH, op.dW, op.ws, peak=peak)
