"""The fine-tuning operators as a training step uses them: layer norm, log-probabilities
through the heads, policy loss, and back through all of them to clipped gradients, against
the same step in 64 bits by automatic differentiation.

Every hand-over is a rounding to the storage type (bf16: 2^-8 of a value): of the normed
states, of dL/dz, of dH, dW, dx.  Each moves a result by at most that share of the sizes
that make it up, and by far less of the norm of a tensor, for the roundings are independent:
the bound is 3 of them on the relative 2-norm.  The loss has fp32 log-probabilities of
bf16 states: 2^-8 of them at most.
"""
import pytest
import torch

import paper_2608_09703_gb300 as mls

pytestmark = pytest.mark.gpu
BF = 2.0 ** -8


def _step(ops, x, gain, bias, W, y, old, ref, adv, start):
    norms, logp, policy, clip = ops
    H = [n.forward(*a) for n, a in zip(norms, zip(x, gain, bias))]
    lp = logp.forward(H, W, y)
    loss = policy(lp, old, adv, y, ref_logp=ref, seq_start=start)
    dH, _ = logp.backward(H, W, y, policy.dlogp)
    for n, a in zip(norms, zip(x, dH, gain)):
        n.backward(*a)
    return loss, clip(1e-3)


def test_a_training_step():
    T, V, d, n = 1500, 2003, (136, 264), 12
    g = torch.Generator(device="cuda").manual_seed(11)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = [(r(T, dm) * 3 + 0.5).bfloat16() for dm in d]
    gain, bias = [(1 + 0.1 * r(dm)).bfloat16() for dm in d], [(0.1 * r(dm)).bfloat16() for dm in d]
    W = [(r(V, dm) * (2.0 / dm ** 0.5)).bfloat16() for dm in d]
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    start = torch.randint(0, T + 1, (n + 1,), generator=g, device="cuda").sort().values.to(torch.int32)
    start[0], start[-1] = 0, T - 30
    t = torch.arange(T, device="cuda")
    seq = (torch.searchsorted(start.long(), t, right=True) - 1).clamp(0, n - 1)
    y[(t - start[seq]) < 20] = -1
    adv = r(n)

    def loss64(x, gain, bias, W, old=None, ref=None):
        rows = []
        for a, gn, b, w in zip(x, gain, bias, W):
            mu = a.mean(1, keepdim=True)
            h = (a - mu) / ((a - mu).square().mean(1, keepdim=True) + 1e-5).sqrt() * gn + b
            lp = torch.log_softmax(h @ w.T, 1)
            rows.append(lp.gather(1, y.clamp(min=0).long()[:, None])[:, 0])
        lp = torch.stack(rows)
        if old is None:
            return lp
        on = (y >= 0) & (t < start[-1])
        ratio = torch.exp(lp - old.double())
        A = adv.double()[seq]
        k = ref.double() - lp
        L = -torch.minimum(ratio * A, ratio.clamp(0.8, 1.2) * A) + 0.05 * (torch.expm1(k) - k)
        cnt = torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, seq, on.double())
        weight = torch.where(on, 1.0 / (n * cnt.clamp(min=1))[seq], 0.0)
        return (L * weight).sum()

    leaves = [[v.double().requires_grad_() for v in group] for group in (x, gain, bias, W)]
    with torch.no_grad():
        lp = loss64(*leaves)
        # off the clipping bounds by 0.05: a rounding of the states moves no token across one
        shift = 0.4 * r(2, T)
        for bound in (0.182, -0.223):
            shift = torch.where((shift - bound).abs() < 0.08, torch.full_like(shift, bound + 0.1), shift)
        old = (lp - shift).float()
        ref = (lp + 0.3 * r(2, T)).float()
    want = loss64(*leaves, old=old, ref=ref)
    want.backward()

    norms = [mls.LayerNorm(T, dm) for dm in d]
    logp = mls.HeadLogp(d, T, V)
    policy = mls.PolicyLoss(T, V, M=2, B=n, beta=0.05, agg="seq", adv_per_seq=True)
    grads = [t for op in norms for t in (op.dx, op.dgain, op.dbias)] + logp.dW
    clip = mls.GradClip(grads)
    ops = (norms, logp, policy, clip)
    loss, stats = _step(ops, x, gain, bias, W, y, old, ref, adv, start)
    size = float(policy.tok_loss.abs().double().sum()) / n
    assert abs(loss.item() - want.item()) <= BF * max(size, abs(want.item()))
    exact = [l.grad for m in range(2) for l in (leaves[0][m], leaves[1][m], leaves[2][m])] + [l.grad for l in leaves[3]]
    total = sum(float(e.square().sum()) for e in exact) ** 0.5
    norm, c = stats.tolist()
    assert abs(norm - total) <= 3 * BF * total and c == pytest.approx(1e-3 / norm, rel=1e-3)
    for got, e in zip(grads, exact):
        assert float((got.double() / c - e).norm()) <= 3 * BF * float(e.norm())
    assert mls.mls_get_status() == 0

    # the whole step captured: same bits on every replay
    first = [g.clone() for g in grads] + [loss.clone(), stats.clone()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            _step(ops, x, gain, bias, W, y, old, ref, adv, start)
    for _ in range(3):
        for g_ in grads:
            g_.fill_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(grads + [loss, stats], first))
