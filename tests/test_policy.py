"""Clipped policy loss with a KL term, and its gradient, against the definition in 64
bits, sequence by sequence.

Tolerances, token by token, with u = 2^-24: the difference D = logp - old is rounded
once (|D| u in the ratio), expf is within 2 units of the last place (4 u) and the
products add a few u, so r A has (|D| + 8) u.  K = e^x - x - 1 comes from its series
below 1/2 (12 u of it), else from expf (6 u of e^x + 1 + |x|), and x is rounded once.
Sums are taken in 32 bits over 8 tokens and in 64 from there: 16 u of the terms' sizes.
"""
import ctypes
import math

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from paper_2608_09703_gb300 import build as mbuild

U = 2.0 ** -24


def reference(c, logp, old, ref, adv, y, start, scale=1.0):
    """Outputs and their tolerances on the CPU, from the formulas."""
    logp, old, adv = logp.double().cpu(), old.double().cpu(), adv.double().cpu()
    ref = None if ref is None else ref.double().cpu()
    y = y.cpu()
    M, T = logp.shape
    lo, hi = 1 - float(torch.tensor(c["clip_low"])), 1 + float(torch.tensor(c["clip_high"]))
    beta = float(torch.tensor(c["beta"]))
    ok = (y >= 0) & (y < c["V"])
    bounds = [(0, T)] if start is None else list(zip(start.tolist()[:-1], start.tolist()[1:]))
    weight, A = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.float64)
    on = torch.zeros(T, dtype=torch.bool)
    for a, b in bounds:
        on[a:b] = ok[a:b]
    N = int(on.sum())
    for i, (a, b) in enumerate(bounds):
        n = int(on[a:b].sum())
        w = {"token": 1 / max(N, 1), "seq": 1 / (len(bounds) * max(n, 1)), "sum": 1.0}[c["agg"]]
        weight[a:b] = torch.where(on[a:b], w, 0.0)
        A[a:b] = adv[i] if c["adv_per_seq"] else adv[a:b]
    A = torch.where(on, A, 0.0)
    D = torch.where(on, logp - old, 0.0)
    r = torch.exp(D)
    stop = ((A > 0) & (r > hi)) | ((A < 0) & (r < lo))
    P = -torch.minimum(r * A, r.clamp(lo, hi) * A)
    P = torch.where(A == 0, 0.0, P)
    g = torch.where(stop | (A == 0), 0.0, -r * A)
    tolP = U * P.abs() * (D.abs() + 8)
    tolg = U * g.abs() * (D.abs() + 8)
    K = torch.zeros_like(P)
    tolK = torch.zeros_like(P)
    if ref is not None:
        x = torch.where(on, ref - logp, 0.0)
        K = torch.expm1(x) - x
        e = torch.exp(x)
        tolK = U * (12 * K + torch.where(x.abs() >= 0.49, 6 * (e + 1 + x.abs()), 0.0)
                    + x.abs() * torch.expm1(x).abs())
        g = g - beta * torch.expm1(x)
        tolg = tolg + beta * U * (16 * torch.expm1(x).abs() + x.abs() * e
                                  + torch.where(x.abs() >= 0.49, 6 * (e + 1), 0.0)) + 2 * U * g.abs()
    L = torch.where(on, P + beta * K, 0.0)
    tolL = tolP + beta * tolK + 4 * U * (P.abs() + beta * K)
    w = torch.tensor([1.0] * M if c["w"] is None else [float(torch.tensor(v)) for v in c["w"]], dtype=torch.float64)
    f = w[:, None] * scale * weight
    tiny = 2.0 ** -149
    total = lambda v: (v * weight).sum(1)  # noqa: E731
    diag = torch.stack([total(P), total(K), total(stop.double())])
    tol_diag = torch.stack([total(tolP + 16 * U * P.abs()), total(tolK + 16 * U * K),
                            16 * U * total(stop.double())]) + 2 * U * diag.abs() + tiny
    out = dict(loss=(w * total(L)).sum().reshape(1), tok_loss=L, diag=diag, dlogp=torch.where(on, g * f, 0.0))
    tol = dict(loss=(w.abs() * total(tolL + 16 * U * (P.abs() + beta * K))).sum().reshape(1)
               + 4 * U * out["loss"].abs() + tiny,
               tok_loss=tolL + tiny, diag=tol_diag, dlogp=tolg * f.abs() + 6 * U * out["dlogp"].abs() + 2 * tiny)
    return out, tol


def config(T, V=1000, M=1, B=0, clip_low=0.2, clip_high=0.28, beta=0.0, agg="token", adv_per_seq=False, w=None):
    return dict(T=T, V=V, M=M, B=B, clip_low=clip_low, clip_high=clip_high, beta=beta, agg=agg,
                adv_per_seq=adv_per_seq, w=w)


def inputs(c, seed=0, lens=None, ignored=0.3):
    g = torch.Generator().manual_seed(seed)
    T, M, n = c["T"], c["M"], c["B"]
    logp = -torch.empty(M, T).exponential_(1.0, generator=g)
    old = logp + 0.3 * torch.randn(M, T, generator=g)
    ref = logp + torch.randn(M, T, generator=g) * torch.where(torch.rand(M, T, generator=g) < 0.5, 1e-3, 0.7)
    y = torch.randint(0, c["V"], (T,), generator=g, dtype=torch.int32)
    y[torch.rand(T, generator=g) < ignored] = -1
    start = None
    if n:
        if lens is None:
            cut = torch.randint(0, T + 1, (n + 1,), generator=g).sort().values
        else:
            cut = torch.tensor([0] + list(lens)).cumsum(0)
        start = cut.to(torch.int32)
    adv = torch.randn(n if c["adv_per_seq"] else T, generator=g)
    return [None if t is None else t.cuda() for t in (logp, old, ref, adv, y, start)]


def run(c, logp, old, ref, adv, y, start, scale=1.0):
    op = mls.PolicyLoss(**c)
    for t in (op.loss, op.tok_loss, op.diag, op.dlogp):
        t.fill_(float("nan"))
    op.ws.fill_(0x7f)
    op(logp, old, adv, y, ref_logp=ref, seq_start=start, grad_scale=scale)
    return op


def check(c, data, scale=1.0):
    op = run(c, *data, scale=scale)
    want, tol = reference(c, *data, scale=scale)
    for k in want:
        err = (getattr(op, k).cpu().double() - want[k]).abs()
        bad = ~(err <= tol[k])
        assert not bad.any(), (k, int(bad.sum()), float((err / tol[k]).nan_to_num(1e9).max()))
    assert mls.mls_get_status() == 0
    return op


@pytest.mark.gpu
@pytest.mark.parametrize("agg", ["token", "seq", "sum"])
@pytest.mark.parametrize("T,n", [(1, 1), (2, 2), (31, 3), (1024, 9), (1025, 2), (2047, 5), (2048, 1), (2049, 40), (4096, 2),
                                 (5000, 4000), (9001, 3), (20011, 300)])
def test_ragged_sequences(T, n, agg):
    c = config(T, B=n, agg=agg, adv_per_seq=T % 2 == 1, beta=0.07, M=1 + T % 3)
    check(c, inputs(c, seed=T))


@pytest.mark.gpu
@pytest.mark.parametrize("agg,n", [("token", 700), ("seq", 700), ("seq", 3), ("sum", 0), ("seq", 200000)])
def test_many_tokens(agg, n):
    """More chunks of tokens than their counts' table has entries of one block; far more sequences than blocks."""
    T = 1100003 if n < 10000 else 1048577
    c = config(T, B=n, agg=agg, beta=0.07, M=2)
    data = inputs(c, seed=n)
    if n >= 10000:  # most of one token or none: too many for the loop of the reference
        op = run(c, *data)
        logp, old, ref, adv, y, start = data
        s = (torch.searchsorted(start.long(), torch.arange(T, device="cuda"), right=True) - 1)
        on = (y >= 0) & (s >= 0) & (s < n)
        s = s.clamp(0, n - 1)
        cnt = torch.zeros(n, device="cuda", dtype=torch.float64).index_add_(0, s, on.double())
        want = torch.where(on, op.tok_loss.double() / (n * cnt.clamp(min=1))[s], 0.0).sum(1)
        got = (op.diag[0].double() + float(torch.tensor(0.07)) * op.diag[1].double())
        size = torch.where(on, op.tok_loss.double().abs() / (n * cnt.clamp(min=1))[s], 0.0).sum(1)
        assert bool(((got - want).abs() <= 32 * U * size).all())
        assert not op.dlogp[:, ~on].any() and not op.tok_loss[:, ~on].any()
        return
    check(c, data)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 77, 2500, 8193])
@pytest.mark.parametrize("agg", ["token", "sum"])
def test_without_sequences(T, agg):
    c = config(T, agg=agg, M=4, w=[1.0, 0.5, -2.0, 0.0])
    data = inputs(c, seed=T)
    data[2] = None  # no reference model
    op = check(c, data, scale=0.125)
    assert not op.diag[1].any()


@pytest.mark.gpu
def test_sequence_borders():
    """Empty sequences in a row, sequences that end at a block's end or cross several, one that is
    all prompt, tokens before the first and behind the last sequence."""
    lens = [0, 0, 2048, 0, 1, 2047, 4097, 0, 3, 5000, 0, 1023, 1]
    T = sum(lens) + 700
    for agg in ("token", "seq", "sum"):
        c = config(T, B=len(lens), agg=agg, adv_per_seq=True, beta=0.1)
        data = inputs(c, seed=3, lens=lens)
        data[4][2048:2049] = -1  # the sequence of one token
        check(c, data)
        data[5] += 300  # tokens in front too
        op = check(c, data)
        start = data[5].tolist()
        for t in (op.tok_loss, op.dlogp):
            assert not t[:, :start[0]].any() and not t[:, start[-1]:].any()


@pytest.mark.gpu
@pytest.mark.parametrize("agg", ["token", "seq", "sum"])
@pytest.mark.parametrize("T", [50, 6000])
def test_nothing_counts(T, agg):
    c = config(T, B=3, agg=agg, beta=0.1)
    data = inputs(c)
    data[4].fill_(-1)
    op = check(c, data)
    assert op.loss.item() == 0 and not op.dlogp.any() and not op.tok_loss.any() and not op.diag.any()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf"), -3.4028234663852886e38])
def test_what_does_not_count_is_not_read(bad):
    c = config(5000, B=7, agg="seq", beta=0.1, M=2, V=500)
    data = inputs(c)
    data[4][100:200] = 500  # a target past the vocabulary does not count either
    off = (data[4] < 0) | (data[4] >= 500)
    want = run(c, *data)
    for k in (0, 1, 2):
        data[k] = torch.where(off, torch.full_like(data[k], bad), data[k])
    data[3] = torch.where(off, torch.full_like(data[3], bad), data[3])
    got = run(c, *data)
    for k in ("loss", "tok_loss", "diag", "dlogp"):
        assert torch.equal(getattr(want, k), getattr(got, k)), k


@pytest.mark.gpu
def test_clipping_bounds_are_exact():
    """Ratios next to a bound, a few units of the last place to either side of it."""
    c = config(4096, clip_low=0.2, clip_high=0.28, agg="sum")
    hi, lo = (math.log(1 + float(torch.tensor(0.28))), math.log(1 - float(torch.tensor(0.2))))
    g = torch.Generator().manual_seed(0)
    old = -torch.empty(1, 4096, dtype=torch.float64).exponential_(2.0, generator=g)
    old = old.float()
    edge = torch.where(torch.arange(4096) % 2 == 0, hi, lo)
    logp = (old.double() + edge).float()
    for _ in range(3):
        step = torch.randint(0, 2, (1, 4096), generator=g) * 2 - 1
        logp = torch.nextafter(logp, logp + step)
    adv = torch.where(torch.arange(4096) % 2 == 0, 1.0, -1.0)
    data = [t.cuda() for t in (logp, old)] + [None, adv.cuda(),
                                              torch.zeros(4096, dtype=torch.int32, device="cuda"), None]
    op = check(c, data)
    D = logp.double() - old.double()
    stopped = torch.where(adv > 0, D > hi, D < lo)[0]
    assert 500 < int(stopped.sum()) < 3600
    assert torch.equal((op.dlogp[0] == 0).cpu(), stopped)


@pytest.mark.gpu
def test_ratios_that_overflow():
    """r = inf: stopped for a gain, an infinite loss for a loss, nothing for an advantage of 0."""
    c = config(8)
    logp = torch.zeros(1, 8, device="cuda")
    old = torch.tensor([[-200.0, -200.0, -200.0, 200.0, 200.0, -float("inf"), -float("inf"), 0.0]], device="cuda")
    adv = torch.tensor([1.0, -1.0, 0.0, 1.0, -1.0, 1.0, 0.0, 0.0], device="cuda")
    y = torch.zeros(8, dtype=torch.int32, device="cuda")
    op = run(c, logp, old, None, adv, y, None)
    L, d = op.tok_loss[0].tolist(), op.dlogp[0].tolist()
    hi, lo = 1 + float(torch.tensor(0.28)), 1 - float(torch.tensor(0.2))
    assert L[0] == pytest.approx(-hi) and d[0] == 0
    assert L[1] == float("inf") and d[1] == float("inf")
    assert L[2] == 0 and d[2] == 0
    assert L[3] == 0 and d[3] == 0  # r = 0 with a gain: P = -0
    assert L[4] == pytest.approx(lo) and d[4] == 0
    assert L[5] == pytest.approx(-hi) and d[5] == 0
    assert L[6] == 0 and d[6] == 0 and L[7] == 0


@pytest.mark.gpu
def test_unbounded_clipping_and_reported_kl():
    c = config(300, clip_low=1.5, clip_high=float("inf"), beta=0.0)
    logp, old, ref, adv, y, start = inputs(c)
    op = run(c, logp, old, ref, adv, y, start)
    on = (y >= 0)
    r = torch.exp(logp.double() - old.double())
    want = torch.where(on, -r * adv, 0.0)
    assert torch.allclose(op.tok_loss.double(), want, rtol=1e-5, atol=1e-30)
    assert op.diag[2].item() == 0
    x = (ref.double() - logp.double())[0][on]
    kl = (torch.expm1(x) - x).mean()
    assert abs(op.diag[1].item() - kl.item()) <= 1e-5 * kl.item()  # reported although beta is 0


@pytest.mark.gpu
def test_gradient_against_differences():
    c = config(400, B=6, agg="seq", beta=0.3, M=2, w=[1.0, 0.4], adv_per_seq=True)
    data = inputs(c, seed=9)
    op = check(c, data)
    g = torch.Generator().manual_seed(1)
    v = torch.randn(2, 400, generator=g, dtype=torch.float64)
    D = (data[0].double() - data[1].double()).cpu()
    for bound in (math.log(1.28), math.log(0.8)):  # no direction across a bound's corner
        v[(D - bound).abs() < 1e-4] = 0
    h = 1e-6
    vals = [reference(c, data[0].double().cpu() + s * h * v, *data[1:])[0]["loss"].item() for s in (1, -1)]
    want, got = (vals[0] - vals[1]) / (2 * h), float((op.dlogp.cpu().double() * v).sum())
    assert abs(got - want) <= 1e-6 * float((op.dlogp.cpu().double() * v).abs().sum()) + 1e-9


@pytest.mark.gpu
def test_outputs_are_optional_and_dlogp_may_replace_logp():
    c = config(5000, B=4, agg="seq", beta=0.1)
    data = inputs(c)
    want = run(c, *data)
    prob = mls.PolicyProblem(**c)
    loss, logp = torch.empty(1, device="cuda"), data[0].clone()
    mls.mls_policy_loss(prob, logp, data[1], data[2], data[3], data[4], data[5], 1.0, loss, None, None, None, want.ws)
    assert torch.equal(loss, want.loss)
    mls.mls_policy_loss(prob, logp, data[1], data[2], data[3], data[4], data[5], 1.0, loss, None, None, logp, want.ws)
    assert torch.equal(loss, want.loss) and torch.equal(logp, want.dlogp)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [500, 7000])
def test_bad_sequence_offsets_are_reported(T):
    """Unsorted offsets or offsets outside the tokens are read within bounds and reported."""
    c = config(T, B=4, agg="seq", adv_per_seq=True)
    data = inputs(c)
    for cut in ([0, 400, 100, 450, 480], [-5, 10, 20, 30, 40], [0, 10, 20, 30, T + 7],
                [2147483647, -2147483648, 0, 3, 1]):
        data[5] = torch.tensor(cut, dtype=torch.int32, device="cuda")
        run(c, *data)
        assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ
    data[5] = torch.tensor([0, 10, 10, 30, 40], dtype=torch.int32, device="cuda")
    check(c, data)


@pytest.mark.gpu
def test_no_tokens():
    c = config(0, B=0)
    e = torch.empty(1, 0, device="cuda")
    op = run(c, e, e, None, torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), None)
    assert op.loss.item() == 0 and not op.diag.any()


@pytest.mark.gpu
@pytest.mark.parametrize("T,n", [(900, 5), (30000, 33)])
def test_repeatable_and_captured(T, n):
    c = config(T, B=n, agg="seq", beta=0.05, M=3)
    sets = [inputs(c, seed=s) for s in (1, 2)]
    ops = [check(c, d) for d in sets]
    want = [[t.clone() for t in (o.loss, o.tok_loss, o.diag, o.dlogp)] for o in ops]
    op, live = ops[0], [t.clone() for t in sets[0]]

    def call():
        op(live[0], live[1], live[3], live[4], ref_logp=live[2], seq_start=live[5])

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call()
    for i in (1, 0, 1, 1):
        for a, b in zip(live, sets[i]):
            a.copy_(b)
        graph.replay()
        got = [t.clone() for t in (op.loss, op.tok_loss, op.diag, op.dlogp)]
        call()  # an eager call right behind it
        again = [t.clone() for t in (op.loss, op.tok_loss, op.diag, op.dlogp)]
        assert all(torch.equal(a, b) for a, b in zip(got, want[i]))
        assert all(torch.equal(a, b) for a, b in zip(again, want[i]))


# ------------------------------------------------------------------ refusals (CPU)
def test_refusals_of_the_library():
    mbuild.build()
    L = B.lib()
    p = 0x1000

    def call(logp=p, old=p, ref=p, adv=p, y=p, start=p, scale=1.0, loss=p, tok=p, dl=0x2000, ws=0x10000,
             size=1 << 30, **kw):
        prob = mls.PolicyProblem(**{**config(100, B=3), **kw})
        return L.mls_policy_loss(prob.ref(), logp, old, ref, adv, y, start, scale, loss, tok, p, dl, ws, size, None)

    for kw in (dict(M=0), dict(M=5), dict(T=-1), dict(T=1 << 31), dict(V=0), dict(V=1 << 31), dict(B=-1),
               dict(clip_low=-0.1), dict(clip_high=float("nan")), dict(beta=-1.0), dict(beta=float("inf")),
               dict(w=[float("nan")]), dict(logp=None), dict(old=None), dict(adv=None), dict(y=None),
               dict(loss=None), dict(dl=p), dict(scale=float("inf")), dict(beta=0.1, ref=None), dict(start=None),
               dict(B=0), dict(B=0, start=None, agg="seq"), dict(B=0, start=None, adv_per_seq=True)):
        assert call(**kw) == B.MLS_ERR_ARG, kw
    for kw in (dict(logp=p + 2), dict(y=p + 1), dict(start=p + 2)):
        assert call(**kw) == B.MLS_ERR_ALIGN, kw
    assert L.mls_policy_loss(None, *[None] * 6, 1.0, *[None] * 5, 0, None) == B.MLS_ERR_ARG
    prob = mls.PolicyProblem(**config(100, B=3))
    prob.c.agg = 7
    assert B.mls_policy_workspace_size(prob) == 0
    assert B.mls_policy_workspace_size(mls.PolicyProblem(**config(1 << 22, B=3))) > 0
    with pytest.raises(KeyError):
        mls.PolicyProblem(100, 10, agg="mean")
    with pytest.raises(ValueError):
        mls.PolicyProblem(100, 10, M=2, w=[1.0])


@pytest.mark.gpu
def test_refusals_of_the_binding():
    c = config(64, B=2)
    logp, old, ref, adv, y, start = inputs(c)
    op = mls.PolicyLoss(**c)
    for kw, err in ((dict(y=y.long()), TypeError), (dict(logp=logp.double()), TypeError),
                    (dict(logp=logp[0]), ValueError), (dict(old=old[:, :63]), ValueError),
                    (dict(adv=adv[:2]), ValueError), (dict(start=start[:2]), ValueError),
                    (dict(old=old.cpu()), ValueError), (dict(ref=ref.t().contiguous().t()[:, :64]), None)):
        a = {**dict(logp=logp, old=old, ref=None, adv=adv, y=y, start=start), **kw}
        if err is None:
            op(a["logp"], a["old"], a["adv"], a["y"], ref_logp=a["ref"], seq_start=a["start"])
            continue
        with pytest.raises(err):
            op(a["logp"], a["old"], a["adv"], a["y"], ref_logp=a["ref"], seq_start=a["start"])
    with pytest.raises(mls.MLSError):
        mls.mls_policy_loss(op.prob, logp, old, None, adv, y, start, 1.0, op.loss, None, None, None, op.ws[:8])


@pytest.mark.gpu
@pytest.mark.parametrize("T,M", [(1, 4), (1024, 2), (3000, 3), (4096, 4), (4097, 4), (200001, 3), (320000, 2)])
def test_models_together_alone_and_in_place(T, M):
    """Every sub-model as by itself, whatever the launch makes of M; dlogp in logp's place; outputs left out."""
    c = config(T, B=3, agg="seq", beta=0.07, M=M, adv_per_seq=True)
    logp, old, ref, adv, y, start = inputs(c, seed=T + M)
    op = run(c, logp, old, ref, adv, y, start)
    total, size = 0.0, 0.0
    for m in range(M):
        one = run(dict(c, M=1), logp[m:m + 1], old[m:m + 1], ref[m:m + 1], adv, y, start)
        assert torch.equal(one.tok_loss[0], op.tok_loss[m]) and torch.equal(one.dlogp[0], op.dlogp[m])
        assert torch.equal(one.diag[:, 0], op.diag[:, m])
        total, size = total + one.loss.item(), size + abs(one.loss.item())
    assert abs(op.loss.item() - total) <= 4 * U * size
    prob = B.PolicyProblem(**c)
    same, loss = logp.clone(), torch.empty(1, device="cuda")
    B.mls_policy_loss(prob, same, old, ref, adv, y, start, 1.0, loss, None, None, same, op.ws)
    assert torch.equal(same, op.dlogp) and torch.equal(loss, op.loss)
    tok = torch.empty_like(logp)
    B.mls_policy_loss(prob, logp, old, ref, adv, y, start, 1.0, loss, tok, None, None, op.ws)
    assert torch.equal(tok, op.tok_loss) and torch.equal(loss, op.loss)
