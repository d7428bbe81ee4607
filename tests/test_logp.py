"""Log-probabilities through the heads and their backward, against the definition in
64 bits.

Tolerances, element by element.  Products of bf16 values are exact in fp32; a sum of d
of them in any order, truncated or rounded at each step, is within 2 d u of the sum of
their sizes (u = 2^-24): E.  Then
  |lse - lse'|   <= E / tau + (2^-22 of the exponential, V / 16 + 64 additions) + 4 u |lse|
  |logp - logp'| <= 2 E / tau + the same
  dL/dz = c (softmax - e_y): each value off by (2 E / tau + 1e-5) of c softmax, then rounded
  to bf16, 2^-8 of it; dH and dW sum those (u for each addition) and are rounded once more.
"""
import ctypes

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from paper_2608_09703_gb300 import build as mbuild

U = 2.0 ** -24
BF = 2.0 ** -8


def inputs(d, T, V, seed=0, ignored=0.2, spread=2.5, zero=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    H = [torch.randn(T, dm, generator=g, device="cuda").bfloat16() for dm in d]
    W = [(torch.randn(V, dm, generator=g, device="cuda") * (spread / dm ** 0.5)).bfloat16() for dm in d]
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    y[torch.rand(T, generator=g, device="cuda") < ignored] = -1
    dl = torch.randn(len(d), T, generator=g, device="cuda")
    dl[torch.rand(len(d), T, generator=g, device="cuda") < zero] = 0
    return H, W, y, dl


def reference(H, W, y, dl, tau):
    out, tol = dict(logp=[], lse=[], dH=[], dW=[]), dict(logp=[], lse=[], dH=[], dW=[])
    tau = float(torch.tensor(tau))
    V = W[0].shape[0]
    ok = (y >= 0) & (y < V)
    idx = torch.where(ok, y, 0).long()[:, None]
    for h, w, g in zip(H, W, dl):
        h, w = h.double(), w.double()
        T, d = h.shape
        z = h @ w.T / tau
        E = 2 * d * U * (h.abs() @ w.abs().T).amax(1) / tau
        lse = torch.logsumexp(z, 1)
        lp = torch.where(ok, z.gather(1, idx)[:, 0] - lse, 0.0)
        add = 2.0 ** -22 + (V / 16 + 64) * U
        t_lse = E + add + 4 * U * (lse.abs() + z.abs().amax(1))
        c = torch.where(ok, g.double() / tau, 0.0)[:, None]
        p = torch.exp(z - lse[:, None])
        G = -c * p
        off = (2 * E[:, None] + 1e-5) * G.abs()
        G = G.scatter_add(1, idx, c)
        off += BF * (G.abs() + off)
        size = G.abs() + off
        dH, dW = G @ w, G.T @ h
        out["lse"].append(lse), out["logp"].append(lp), out["dH"].append(dH), out["dW"].append(dW)
        tol["lse"].append(t_lse), tol["logp"].append(t_lse + E)
        tol["dH"].append(off @ w.abs() + 2 * V * U * (size @ w.abs()) + 1.01 * BF * dH.abs() + 1e-37)
        tol["dW"].append(off.T @ h.abs() + 2 * T * U * (size.T @ h.abs()) + 1.01 * BF * dW.abs() + 1e-37)
    return out, tol


def check(H, W, y, dl, tau=1.0, vocab_group=0, op=None, status=0):
    d, T, V = [w.shape[1] for w in W], H[0].shape[0], W[0].shape[0]
    op = op or mls.HeadLogp(d, T, V, tau=tau, vocab_group=vocab_group)
    for t in [op.logp, op.lse] + op.dH + op.dW:
        t.fill_(float("nan"))
    op.ws.fill_(0xff)
    op.forward(H, W, y)
    op.ws.fill_(0xff)
    op.backward(H, W, y, dl)
    want, tol = reference(H, W, y, dl, tau)
    for k in want:
        for m in range(len(d)):
            got = getattr(op, k)[m]
            err = (got.double() - want[k][m]).abs()
            bad = ~(err <= tol[k][m])
            assert not bad.any(), (k, m, int(bad.sum()), float((err / tol[k][m]).nan_to_num(1e9).max()))
    assert mls.mls_get_status() == status
    return op


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", [
    (1, (64,), 1), (1, (8,), 7), (3, (136,), 300), (17, (64, 200), 255), (128, (72,), 1000), (129, (64, 8, 24), 257),
    (256, (128, 256), 1024), (257, (64,), 1025), (300, (264,), 5003), (513, (64, 72, 80, 200), 777),
    (1000, (520,), 2000), (70, (64, 136), 20000), (2000, (64,), 513)])
def test_against_the_definition(T, d, V):
    check(*inputs(d, T, V, seed=T + V))


@pytest.mark.gpu
@pytest.mark.parametrize("tau", [0.5, 0.7, 1.7, 10.0])
def test_temperature(tau):
    check(*inputs((128, 136), 150, 1500, seed=3), tau=tau)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V,group", [(300, (64, 136), 3000, 768), (513, (72,), 1025, 256),
                                         (40, (264,), 9000, 2048), (1300, (64,), 2100, 1024)])
def test_vocabulary_groups(T, d, V, group):
    """dH adds up over several groups; it is rounded once, at the end."""
    check(*inputs(d, T, V, seed=T), vocab_group=group)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V", [(2700, (264, 776), 33000), (1100, (320, 1008), 33000)])
def test_wide_units_and_split_reductions(T, d, V):
    check(*inputs(d, T, V, seed=T))


@pytest.mark.gpu
def test_tokens_left_out():
    H, W, y, dl = inputs((64, 136), 200, 900, ignored=0.0)
    y[::3], y[1] = -1, 900  # one past the vocabulary: reported and left out
    off = (y < 0) | (y >= 900)
    dl[:, off] = float("nan")  # not used
    op = check(H, W, y, torch.where(off, 0.0, dl), status=B.MLS_STATUS_BAD_TARGET)
    want = [t.clone() for t in op.dH + op.dW]
    op.forward(H, W, y)
    op.backward(H, W, y, dl)
    assert all(torch.equal(a, b) for a, b in zip(op.dH + op.dW, want))
    assert not any(t[off].any() for t in op.dH) and not op.logp[:, off].any()
    mls.mls_get_status()
    y.fill_(-1)
    op.forward(H, W, y)
    op.backward(H, W, y, dl)
    assert not any(t.any() for t in op.dH + op.dW) and not op.logp.any()
    assert torch.isfinite(op.lse).all()


@pytest.mark.gpu
def test_peaked_rows():
    """A token with nearly all of the mass, and one with nearly none."""
    H, W, y, dl = inputs((64,), 64, 500, spread=20.0, ignored=0.0)
    z = H[0].double() @ W[0].double().T
    y[:32], y[32:] = z.argmax(1)[:32].int(), z.argmin(1)[32:].int()
    check(H, W, y, dl)


@pytest.mark.gpu
def test_agrees_with_the_loss():
    """-logp is the loss's cross-entropy, and its gradient with dlogp = -1/N the loss's."""
    H, W, y, _ = inputs((128, 264), 700, 3001, seed=8)
    loss = mls.HeadLoss((128, 264), 700, 3001, alpha=0.0)
    loss.forward(H, W, y)
    op = mls.HeadLogp((128, 264), 700, 3001)
    logp = op.forward(H, W, y)
    assert torch.allclose(-logp, loss.tok_diag[0], rtol=2e-5, atol=2e-5)
    loss.backward(H, W, y)
    dl = torch.full((2, 700), -1.0 / int((y >= 0).sum()), device="cuda")
    dH, dW = op.backward(H, W, y, dl)
    for a, b in zip(dH + dW, loss.dH + loss.dW):
        assert float((a.float() - b).norm() / b.norm()) < BF


@pytest.mark.gpu
def test_gradient_against_differences():
    """Central differences of the definition in 64 bits, along random directions."""
    H, W, y, dl = inputs((64, 40), 48, 300, seed=2)
    op = check(H, W, y, dl, tau=0.8)
    g = torch.Generator(device="cuda").manual_seed(3)
    tau, ok = float(torch.tensor(0.8)), y >= 0

    def value(h, w, c):
        lp = torch.log_softmax(h @ w.T / tau, 1)
        return float((lp.gather(1, y.clamp(min=0).long()[:, None])[:, 0] * torch.where(ok, c.double(), 0.0)).sum())

    for m in range(2):
        for grad, which in ((op.dH[m], 0), (op.dW[m], 1)):
            args = [H[m].double(), W[m].double()]
            v = torch.randn(args[which].shape, generator=g, device="cuda", dtype=torch.float64)
            ends = []
            for s in (1e-5, -1e-5):
                a = list(args)
                a[which] = a[which] + s * v
                ends.append(value(*a, dl[m]))
            want, got = (ends[0] - ends[1]) / 2e-5, float((grad.double() * v).sum())
            # two roundings to bf16, of dL/dz and of the result; random directions
            assert abs(got - want) <= 2 * BF * float((grad.double() * v).norm()) * 3 + 1e-6


@pytest.mark.gpu
def test_no_tokens():
    op = mls.HeadLogp((64,), 0, 100)
    H, W = [torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")], inputs((64,), 1, 100)[1]
    y = torch.empty(0, dtype=torch.int32, device="cuda")
    op.forward(H, W, y)
    op.dW[0].fill_(3.0)
    op.backward(H, W, y, torch.empty(1, 0, device="cuda"))
    assert not op.dW[0].any()


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V,group", [(300, (64, 136), 3000, 768), (70, (64, 136), 20000, 0),
                                         (513, (64, 136), 1000, 0)])
def test_back_to_back_and_captured(T, d, V, group):
    sets = [inputs(d, T, V, seed=s) for s in (1, 2)]
    op = mls.HeadLogp(d, T, V, vocab_group=group)

    def call(x):
        op.forward(*x[:3])
        op.backward(*x)

    outputs = lambda: [t.clone() for t in [op.logp, op.lse] + op.dH + op.dW]  # noqa: E731
    want = []
    for x in sets:
        call(x)
        torch.cuda.synchronize()
        want.append(outputs())
    live = [[t.clone() for t in sets[0][0]], [t.clone() for t in sets[0][1]], sets[0][2].clone(), sets[0][3].clone()]

    def load(x):
        for a, b in zip(live[0] + live[1] + live[2:], x[0] + x[1] + [x[2], x[3]]):
            a.copy_(b)

    got = []
    for i in range(12):
        load(sets[i % 2])
        call(live)
        got.append(outputs())
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, want[i % 2])), i
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call(live)
    for i in (1, 0, 1):
        load(sets[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs(), want[i]))
    assert mls.mls_get_status() == 0


# ------------------------------------------------------------------ refusals (CPU)
def test_refusals_of_the_library():
    mbuild.build()
    L = B.lib()
    p = 0x1000

    def arr(M, v):
        return (ctypes.c_void_p * M)(*([v] * M))

    def call(d=(64, 64), T=10, V=100, h=p, w=p, y=p, lse=p, dl=p, dh=p, dw=p, bwd=True, **kw):
        prob = mls.Problem(d, T, V, **kw)
        M = len(d)
        ws, size = 0x10000, 1 << 40
        if bwd:
            return L.mls_head_logp_bwd(prob.ref(), arr(M, h), arr(M, w), y, lse, dl, arr(M, dh), arr(M, dw), ws, size, None)
        return L.mls_head_logp_fwd(prob.ref(), arr(M, h), arr(M, w), y, dl, lse, ws, size, None)

    for bwd in (False, True):
        for kw in (dict(tau=0.0), dict(tau=float("nan")), dict(d=(64,) * 5), dict(T=-1), dict(V=0), dict(h=None),
                   dict(w=None), dict(y=None), dict(lse=None), dict(dl=None), dict(vocab_group=100)):
            assert call(bwd=bwd, **kw) == B.MLS_ERR_ARG, kw
        assert call(bwd=bwd, d=(64, 60)) == B.MLS_ERR_UNSUPPORTED
        assert call(bwd=bwd, in_dtype=B.MLS_FP32) == B.MLS_ERR_UNSUPPORTED
        for kw in (dict(h=p + 8), dict(w=p + 4), dict(y=p + 2), dict(lse=p + 1)):
            assert call(bwd=bwd, **kw) == B.MLS_ERR_ALIGN, kw
    assert call(dh=None) == B.MLS_ERR_ARG and call(dw=p + 8) == B.MLS_ERR_ALIGN
    # one buffer for both sub-models' gradients, or for a gradient and an input
    q = 0x100000
    assert call(dh=q, dw=2 * q) == B.MLS_ERR_ARG
    for kw in (dict(dh=p, dw=q), dict(dh=q, dw=p), dict(dh=q, dw=q), dict(dh=q, dw=2 * q, h=q)):
        assert call(d=(64,), **kw) == B.MLS_ERR_ARG, kw
    assert L.mls_head_logp_fwd(None, None, None, None, None, None, None, 0, None) == B.MLS_ERR_ARG
    assert B.mls_logp_workspace_size(mls.Problem((64,), 10, 100, in_dtype=B.MLS_FP32)) == 0
    assert B.mls_logp_workspace_size(mls.Problem((64,), 10, 100)) > 0


@pytest.mark.gpu
def test_refusals_of_the_binding():
    H, W, y, dl = inputs((64, 72), 20, 50)
    op = mls.HeadLogp((64, 72), 20, 50)
    op.forward(H, W, y)
    for a, err in (((H, W, y.long()), TypeError), (([h.float() for h in H], W, y), TypeError),
                   ((H[:1], W, y), ValueError), ((H, W[::-1], y), ValueError), ((H, W, y[:19]), ValueError),
                   (([H[0], H[1].t().contiguous().t()], W, y), ValueError), ((H, [W[0].cpu(), W[1]], y), ValueError)):
        with pytest.raises(err):
            op.forward(*a)
    with pytest.raises(ValueError):
        op.backward(H, W, y, dl[:1])
    with pytest.raises(mls.MLSError) as e:
        mls.mls_head_logp_fwd(op.prob, H, W, y, op.logp, op.lse, op.ws[:256])
    assert e.value.code == B.MLS_ERR_WORKSPACE
