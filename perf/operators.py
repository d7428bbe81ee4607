"""Reinforcement fine-tuning of a suite's output stage: the operators between a sub-model's
last hidden state and the optimizer, each in a plain form and through the package.

  norm    layer norm before a head, forward or forward and backward
  logp    log-probabilities of given tokens through the heads, with the backward of a
          gradient per token; the [T, V] logits are never stored
  policy  clipped policy loss with a KL term over ragged sequences, and its gradient
  clip    global gradient norm over many tensors, and clipping in place

A case is a dict of plain values; widths are comma-separated texts.  ``listed`` gives fixed
ones, ``draw`` more of the same ranges.  Where ``own`` is false everything is computed with
elementary torch operations.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
Z_STD = 2.5          # spread of the logits
CLIP_EPS = 1e-6      # added to the norm before the division
DECAY = 0.9999       # of the clipping bound from one call to the next


def _ints(text):
    return [int(x) for x in str(text).split(",")]


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


# ------------------------------------------------------------------------- cases
def listed():
    def norm(name, T, d, dtype="bf16", backward=True, gain=True, bias=True):
        return dict(name=name, kind="norm", T=T, d=d, dtype=dtype, backward=backward, gain=gain, bias=bias)

    def logp(name, T, d, V, tau=1.0, ignored=0.0):
        return dict(name=name, kind="logp", T=T, d=d, V=V, tau=tau, ignored=ignored)

    def policy(name, T, B, M=1, agg="token", per_seq=False, beta=0.0):
        return dict(name=name, kind="policy", T=T, B=B, M=M, agg=agg, per_seq=per_seq, beta=beta,
                    V=50304, prompt=0.3)

    def clip(name, n, total, dtype, scale=True, packed=False):
        return dict(name=name, kind="clip", n=n, total=total, dtype=dtype, scale=scale, packed=packed)

    return [
        # The positions of one user's verify round before the head: latency of interactive decoding.
        norm("norm_decode", 7, 1024, backward=False),
        # A training batch of four packed sequences of 2048 tokens at the middle sub-model's width.
        norm("norm_train", 8192, 2048),
        # The largest batch of the benchmark at the second width of its four-level suite.
        norm("norm_big", 65536, 4096),
        # A fine-tuning micro-batch of nothing round, kept in fp32, a norm with a gain alone.
        norm("norm_ragged", 1531, 1000, "fp32", bias=False),
        # A unit test's suite: latency and the number of launches count.
        logp("logp_tiny", 256, "128,256", 1024),
        # The rollouts of one micro-batch through the two smaller sub-models of the benchmark's suite.
        logp("logp_suite", 4096, "1024,2048", 50304),
        # Nothing round: odd tokens and vocabulary, widths that end inside a tile, the sampling
        # temperature of the rollouts, prompts left out.
        logp("logp_ragged", 1531, "520,1032", 32003, tau=0.7, ignored=0.3),
        # One prompt's group of short answers: latency.
        policy("policy_group", 2000, 8, per_seq=True),
        # A step's rollouts for two sub-models, a mean over sequences, with the KL term.
        policy("policy_batch", 131072, 256, M=2, agg="seq", per_seq=True, beta=0.04),
        # The largest: a four-level suite, 2000 and more long rollouts, an advantage per token.
        policy("policy_large", 4000001, 2048, M=4, agg="token", beta=0.01),
        # The gradients of a small model, flat buckets without padding: latency.
        clip("clip_small", 21, 300007, "mixed", packed=True),
        # The gradients of a model of 1.2 billion parameters.
        clip("clip_model", 200, 1200000000, "bf16"),
    ]


_MOST_FLOPS = 3.8e12    # of logp_suite
_MOST_NORM = 65536 * 4096
_MOST_CLIP = 1200000000


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "logp", "logp", "policy", "policy", "clip"])
    if kind == "norm":
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        while True:
            T, d = _log_int(rng, 1, 65536), 8 * _log_int(rng, 8, 2048)
            if T * d * (2 if dtype == "fp32" else 1) <= _MOST_NORM:
                break
        return dict(kind=kind, T=T, d=d, dtype=dtype, backward=rng.random() < 0.7,
                    gain=rng.random() < 0.9, bias=rng.random() < 0.6)
    if kind == "logp":
        M = rng.choice([1, 1, 2, 3])
        while True:
            d = [8 * _log_int(rng, 8, 1024) for _ in range(M)]
            T, V = _log_int(rng, 1, 16384), _log_int(rng, 500, 256000)
            if 6 * T * V * sum(d) <= _MOST_FLOPS:
                break
        return dict(kind=kind, T=T, d=",".join(map(str, sorted(d))), V=V,
                    tau=rng.choice([1.0, 1.0, round(rng.uniform(0.6, 1.5), 2)]),
                    ignored=rng.choice([0.0, 0.1, 0.5]))
    if kind == "policy":
        M, T = rng.choice([1, 1, 2, 3, 4]), _log_int(rng, 1, 4000000)
        agg = rng.choice(["token", "seq", "sum"])
        per_seq = rng.random() < 0.5
        B = 0 if agg != "seq" and not per_seq and rng.random() < 0.3 else _log_int(rng, 1, min(T, 4096))
        return dict(kind=kind, T=T, B=B, M=M, agg=agg, per_seq=per_seq,
                    beta=rng.choice([0.0, round(rng.uniform(0.01, 0.2), 3)]), V=_log_int(rng, 500, 256000),
                    prompt=rng.choice([0.0, 0.3, 0.6]))
    n = _log_int(rng, 1, 300)
    return dict(kind=kind, n=n, total=_log_int(rng, max(64, n), _MOST_CLIP // 2),
                dtype=rng.choice(["bf16", "fp32", "mixed"]), scale=rng.random() < 0.8,
                packed=rng.random() < 0.5)


# ------------------------------------------------------------------------- inputs
def _gen(seed, k):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 8 + k)
    return g


def _norm_inputs(case, seed):
    """Hidden states with a few channels that stand out and a mean of their own, as a residual
    stream has them, and the gradient that comes back."""
    T, d, dt, g = case["T"], case["d"], _dtype(case), _gen(seed, 0)
    out = torch.where(torch.rand(d, generator=g, device=DEV) < 0.01, 20.0, 1.0)
    x = torch.randn(T, d, generator=g, device=DEV).mul_(out).add_(0.3).to(dt)
    dy = torch.randn(T, d, generator=g, device=DEV).mul_(1e-3).to(dt)
    gain = (1 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(dt) if case["gain"] else None
    bias = (0.1 * torch.randn(d, generator=g, device=DEV)).to(dt) if case["bias"] else None
    return x, gain, bias, dy


def _logp_inputs(case, seed):
    """Normalised hidden states, heads whose logits spread as a trained model's do, the rollouts'
    tokens, prompts left out, and dL/dlogp, which is zero for the clipped tokens."""
    d, T, V, g = _ints(case["d"]), case["T"], case["V"], _gen(seed, 0)
    H = [torch.randn(T, dm, generator=g, device=DEV).bfloat16() for dm in d]
    W = [(torch.randn(V, dm, generator=g, device=DEV) * (Z_STD / math.sqrt(dm))).bfloat16() for dm in d]
    y = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    y = torch.where(torch.rand(T, generator=g, device=DEV) < case["ignored"], -1, y).to(torch.int32)
    dl = torch.randn(len(d), T, generator=g, device=DEV) / T
    dl = torch.where(torch.rand(len(d), T, generator=g, device=DEV) < 0.1, 0.0, dl)
    return H, W, y, dl


def _policy_inputs(case, seed):
    """Rollouts of ragged lengths, each with its prompt left out (a few are nothing else), padding
    behind the last one; log-probabilities that moved a little since the rollout, some far."""
    T, B, M, g = case["T"], case["B"], case["M"], _gen(seed, 0)
    y = torch.randint(0, case["V"], (T,), generator=g, device=DEV, dtype=torch.int32)
    start = None
    t = torch.arange(T, device=DEV)
    if B > 0:
        cut = torch.randint(0, T - T // 50 + 1, (B + 1,), generator=g, device=DEV).sort().values
        cut[0], cut[-1] = 0, T - T // 50
        start = cut.to(torch.int32)
        s = (torch.searchsorted(cut, t, right=True) - 1).clamp(max=B - 1)
        part = case["prompt"] * (0.5 + torch.rand(B, generator=g, device=DEV))
        part = torch.where(torch.rand(B, generator=g, device=DEV) < 0.02, 1.0, part)
        y = torch.where((t - cut[s]) < part[s] * (cut[s + 1] - cut[s]), -1, y)
    else:
        y = torch.where(torch.rand(T, generator=g, device=DEV) < case["prompt"], -1, y)
    logp = torch.empty(M, T, device=DEV).exponential_(1.0, generator=g).neg_()
    far = torch.where(torch.rand(M, T, generator=g, device=DEV) < 0.02, 1.0, 0.1)
    old = logp + far * torch.randn(M, T, generator=g, device=DEV)
    ref = logp + 0.2 * torch.randn(M, T, generator=g, device=DEV)
    adv = torch.randn(B if case["per_seq"] else T, generator=g, device=DEV)
    return logp, old, (ref if case["beta"] > 0 else None), adv, y.to(torch.int32), start


def _clip_sizes(case):
    """Sizes of the tensors: some few hold most of the values, many are norms' and biases'."""
    rng = random.Random(case["n"] * 1000003 + case["total"])
    share = [math.exp(rng.gauss(0.0, 2.0)) for _ in range(case["n"])]
    left = case["total"] - case["n"]
    return [1 + int(left * s / sum(share)) for s in share], [
        case["dtype"] if case["dtype"] != "mixed" else rng.choice(["bf16", "fp32"]) for _ in share], [
        10 ** rng.uniform(-4, -1) for _ in share]


def _clip_inputs(case, seed):
    """Gradients of many tensors in one flat buffer per type, each tensor a view of it: without
    padding (packed), or each on a boundary of 256 bytes."""
    sizes, types, sigma = _clip_sizes(case)
    flat, views = {}, []
    for k, name in enumerate(("bf16", "fp32")):
        pad = 1 if case["packed"] else 256 // (2 if name == "bf16" else 4)
        at = [0]
        for n, ty in zip(sizes, types):
            at.append(at[-1] + (-(-n // pad) * pad if ty == name else 0))
        if at[-1] == 0:
            continue
        dt = torch.bfloat16 if name == "bf16" else torch.float32
        buf, g = torch.zeros(at[-1], device=DEV, dtype=dt), _gen(seed, k)
        flat[name] = buf
        for i, (n, ty, s) in enumerate(zip(sizes, types, sigma)):
            if ty == name:
                v = buf[at[i]:at[i] + n]
                v.normal_(0.0, s, generator=g)
                views.append((i, v))
    views = [v for _, v in sorted(views, key=lambda x: x[0])]
    norm = math.sqrt(sum(n * s * s for n, s in zip(sizes, sigma)))
    return flat, views, (0.37 * norm if case["scale"] else math.inf)


# ------------------------------------------------------------------------- passes
def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case, "kind": kind}
    s["in"] = {"norm": _norm_inputs, "logp": _logp_inputs, "policy": _policy_inputs,
               "clip": _clip_inputs}[kind](case, seed)
    if kind == "clip":
        s["max"] = s["in"][2]
    if own:  # the handle with its outputs and workspace, kept from step to step
        import paper_2608_09703_gb300 as mls

        if kind == "norm":
            s["op"] = mls.LayerNorm(case["T"], case["d"], gain=case["gain"], bias=case["bias"],
                                    dtype=_dtype(case), device=DEV, backward=case["backward"])
        elif kind == "logp":
            s["op"] = mls.HeadLogp(_ints(case["d"]), case["T"], case["V"], tau=case["tau"], device=DEV)
        elif kind == "policy":
            s["op"] = mls.PolicyLoss(case["T"], case["V"], M=case["M"], B=case["B"], clip_low=0.2,
                                     clip_high=0.28, beta=case["beta"], agg=case["agg"],
                                     adv_per_seq=case["per_seq"], device=DEV)
        else:
            s["op"] = mls.GradClip(s["in"][1])
    return s


def run(s):
    if own:
        return _run_own(s)
    return {"norm": _plain_norm, "logp": _plain_logp, "policy": _plain_policy, "clip": _plain_clip}[s["kind"]](s)


def _run_own(s):
    kind, op = s["kind"], s["op"]
    if kind == "norm":
        x, gain, bias, dy = s["in"]
        got = {"y": op.forward(x, gain, bias)}
        if s["case"]["backward"]:
            got["dx"], got["dgain"], got["dbias"] = op.backward(x, dy, gain)
        return got
    if kind == "logp":
        H, W, y, dl = s["in"]
        logp = op.forward(H, W, y)
        dH, dW = op.backward(H, W, y, dl)
        return {"logp": logp, "lse": op.lse, "dH": dH, "dW": dW}
    if kind == "policy":
        logp, old, ref, adv, y, start = s["in"]
        loss = op(logp, old, adv, y, ref_logp=ref, seq_start=start)
        return {"loss": loss, "tok_loss": op.tok_loss, "diag": op.diag, "dlogp": op.dlogp}
    # A bound that shrinks a little from call to call: the gradients, clipped in place, are
    # over it again, so that every call has the same work.
    stats = op(s["max"])
    s["max"] *= DECAY
    return {"stats": stats, "grads": s["in"][0]}


def _plain_norm(s):
    x, gain, bias, dy = s["in"]
    dt, d = x.dtype, x.shape[1]
    xf = x.float()
    c = xf - xf.mean(1, keepdim=True)
    r = torch.rsqrt((c * c).mean(1, keepdim=True) + 1e-5)
    xh = c * r
    g = torch.ones(d, device=DEV) if gain is None else gain.float()
    y = xh * g if bias is None else xh * g + bias.float()
    got = {"y": y.to(dt)}
    if s["case"]["backward"]:
        dyf = dy.float()
        gy = dyf * g
        dx = r * (gy - gy.mean(1, keepdim=True) - xh * (gy * xh).mean(1, keepdim=True))
        got["dx"] = dx.to(dt)
        got["dgain"] = None if gain is None else (dyf * xh).sum(0)
        got["dbias"] = None if bias is None else dyf.sum(0)
    return got


def _plain_logp_one(H, W, y, dl, tau):
    ok = y >= 0
    idx = y.clamp(min=0).long()[:, None]
    Hf, Wf = H.float(), W.float()
    z = (Hf @ Wf.T) / tau
    top = z.max(1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    logp = torch.where(ok, (z.gather(1, idx) - lse)[:, 0], 0.0)
    c = torch.where(ok, dl / tau, 0.0)[:, None]
    G = e.mul_(-c / total).scatter_add_(1, idx, c)
    return logp, lse[:, 0], (G @ Wf).to(H.dtype), (G.T @ Hf).to(W.dtype)


def _plain_logp(s):
    H, W, y, dl = s["in"]
    tau = s["case"]["tau"]
    got = [_plain_logp_one(h, w, y, g, tau) for h, w, g in zip(H, W, dl)]
    return {"logp": torch.stack([x[0] for x in got]), "lse": torch.stack([x[1] for x in got]),
            "dH": [x[2] for x in got], "dW": [x[3] for x in got]}


def _sequences(case, start, counted):
    """Per token its sequence (0 where there is none) and whether it counts; per sequence its counted tokens."""
    T, B = case["T"], case["B"]
    if B == 0:
        return torch.zeros(T, dtype=torch.int64, device=DEV), counted, None
    t = torch.arange(T, device=DEV)
    s = torch.searchsorted(start.long(), t, right=True) - 1
    counted = counted & (s >= 0) & (s < B)
    s = s.clamp(0, B - 1)
    n = torch.zeros(B, device=DEV, dtype=torch.float64).index_add_(0, s, counted.double())
    return s, counted, n


def _policy(case, inputs, f):
    """The loss in the type f; the difference that the clipping goes by in 64 bits."""
    logp, old, ref, adv, y, start = inputs
    s, counted, n = _sequences(case, start, (y >= 0) & (y < case["V"]))
    if case["agg"] == "token":
        weight = counted.to(f) / counted.sum().clamp(min=1).to(f)
    elif case["agg"] == "seq":
        weight = torch.where(counted, 1.0 / (case["B"] * n[s].clamp(min=1)), 0.0).to(f)
    else:
        weight = counted.to(f)
    A = (adv[s] if case["per_seq"] else adv).to(f)[None, :]
    delta = logp.double() - old.double()
    r = torch.exp(delta.to(f))
    over = (A > 0) & (torch.exp(delta) > 1 + 0.28)
    under = (A < 0) & (torch.exp(delta) < 1 - 0.2)
    part = torch.where(over, -(1 + 0.28) * A, torch.where(under, -(1 - 0.2) * A, -r * A))
    grad = torch.where(over | under, 0.0, -r * A)
    kl = torch.zeros_like(part)
    if ref is not None:
        x = (ref.double() - logp.double())
        kl = (torch.expm1(x) - x).to(f)
        grad = grad - case["beta"] * torch.expm1(x).to(f)
    c = counted[None, :]
    tok = torch.where(c, part + case["beta"] * kl, 0.0)
    diag = [torch.where(c, v.to(f) * weight, 0.0).sum(1, dtype=torch.float64) for v in (part, kl, over | under)]
    loss = torch.where(c, tok * weight, 0.0).sum(dtype=torch.float64)
    return {"loss": loss.reshape(1).to(f), "tok_loss": tok, "diag": torch.stack(diag).to(f),
            "dlogp": torch.where(c, grad * weight, 0.0)}


def _plain_policy(s):
    return _policy(s["case"], s["in"], torch.float32)


def _plain_clip(s):
    flat, views, _ = s["in"]
    most = s["max"]
    s["max"] = most * DECAY
    norm = torch.stack([v.float().square().sum(dtype=torch.float64) for v in views]).sum().sqrt().float()
    if math.isinf(most):
        return {"stats": torch.stack([norm, torch.ones_like(norm)]), "grads": flat}
    coef = (most / (norm + CLIP_EPS)).clamp(max=1.0)
    [v.copy_(v.float() * coef) for v in views]
    return {"stats": torch.stack([norm, coef]), "grads": flat}


def work(case):
    """Each input read once, each output written once, and the products and sums that the
    definitions need (a logp pass: the logits, dH and dW)."""
    kind = case["kind"]
    if kind == "norm":
        T, d, elt = case["T"], case["d"], 4 if case["dtype"] == "fp32" else 2
        few = d * elt * (case["gain"] + case["bias"])
        if case["backward"]:  # x, dy, y, dx, the row statistics handed on
            return {"bytes": 4 * T * d * elt + 16 * T + few + 4 * d * (case["gain"] + case["bias"]),
                    "flops": 22 * T * d}
        return {"bytes": 2 * T * d * elt + few, "flops": 8 * T * d}
    if kind == "logp":
        T, V, d = case["T"], case["V"], _ints(case["d"])
        return {"bytes": 4 * (T + V) * sum(d) + 4 * T + 12 * T * len(d), "flops": 6 * T * V * sum(d)}
    if kind == "policy":
        T, M = case["T"], case["M"]
        rows = 4 * T * M * (4 + (case["beta"] > 0))
        return {"bytes": rows + 4 * T + 4 * (case["B"] if case["per_seq"] else T) + 4 * (case["B"] + 1),
                "flops": 20 * T * M}
    sizes, types, _ = _clip_sizes(case)
    size = sum(n * (4 if ty == "fp32" else 2) for n, ty in zip(sizes, types))
    return {"bytes": size * (2 if case["scale"] else 1), "flops": sum(sizes) * (3 if case["scale"] else 2)}


# ------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    return {"norm": _exact_norm, "logp": _exact_logp, "policy": _exact_policy, "clip": _exact_clip}[case["kind"]](case, seed)


def _exact_norm(case, seed):
    x, gain, bias, dy = _norm_inputs(case, seed)
    T, d = x.shape
    g = torch.ones(d, device=DEV, dtype=torch.float64) if gain is None else gain.double()
    y = torch.empty_like(x, dtype=torch.float64)
    dx = torch.empty_like(y) if case["backward"] else None
    dgain, dbias = torch.zeros_like(g), torch.zeros_like(g)
    step = max(1, (1 << 24) // d)
    for a in range(0, T, step):
        xd, gd = x[a:a + step].double(), dy[a:a + step].double()
        var, mean = torch.var_mean(xd, 1, correction=0, keepdim=True)
        sd = torch.sqrt(var + 1e-5)
        xh = (xd - mean) / sd
        y[a:a + step] = xh * g + (0.0 if bias is None else bias.double())
        if case["backward"]:
            dgain += torch.einsum("td,td->d", gd, xh)
            dbias += gd.sum(0)
            gd = gd * g
            along = torch.einsum("td,td->t", gd, xh)[:, None] / d
            dx[a:a + step] = (gd - gd.sum(1, keepdim=True) / d - xh * along) / sd
    got = {"y": y}
    if case["backward"]:
        got.update(dx=dx, dgain=dgain if case["gain"] else None, dbias=dbias if case["bias"] else None)
    return got


def _exact_logp(case, seed):
    H, W, y, dl = _logp_inputs(case, seed)
    T, V, tau = case["T"], case["V"], case["tau"]
    got = {"logp": torch.zeros(len(H), T, device=DEV, dtype=torch.float64), "dH": [], "dW": []}
    got["lse"] = torch.zeros_like(got["logp"])
    step = max(1, (1 << 26) // V)
    for m in range(len(H)):
        Hd, Wd = H[m].double(), W[m].double()
        dH, dW = torch.zeros_like(Hd), torch.zeros_like(Wd)
        for a in range(0, T, step):
            yc = y[a:a + step].long()
            ok = yc >= 0
            lp = torch.log_softmax(Hd[a:a + step] @ Wd.T / tau, 1)
            z = (Hd[a:a + step] * Wd[yc.clamp(min=0)]).sum(1) / tau
            own_lp = lp.gather(1, yc.clamp(min=0)[:, None])[:, 0]
            got["lse"][m, a:a + step] = z - own_lp
            got["logp"][m, a:a + step] = torch.where(ok, own_lp, 0.0)
            G = -lp.exp_()
            G[torch.arange(len(yc), device=DEV), yc.clamp(min=0)] += 1.0
            G *= torch.where(ok, dl[m, a:a + step].double() / tau, 0.0)[:, None]
            dH[a:a + step] = G @ Wd
            dW += G.T @ Hd[a:a + step]
        got["dH"].append(dH)
        got["dW"].append(dW)
    return got


def _exact_policy(case, seed):
    """Sequence by sequence from the definition where there are few, else by running sums."""
    logp, old, ref, adv, y, start = [None if v is None else v.double() if v.is_floating_point() else v.long()
                                     for v in _policy_inputs(case, seed)]
    T, B = case["T"], case["B"]
    y = y.clone()
    bounds = torch.tensor([0, T], device=DEV) if start is None else start
    y[: int(bounds[0])] = -1
    y[int(bounds[-1]):] = -1
    ok = (y >= 0) & (y < case["V"])
    upto = torch.cat([torch.zeros(1, device=DEV, dtype=torch.int64), ok.long().cumsum(0)])
    n = upto[bounds[1:]] - upto[bounds[:-1]]
    lens = bounds[1:] - bounds[:-1]
    seq = torch.repeat_interleave(torch.arange(len(lens), device=DEV), lens)
    first = int(bounds[0])
    per = torch.zeros(T, device=DEV, dtype=torch.float64)
    if case["agg"] == "seq":
        per[first:first + len(seq)] = 1.0 / (B * n.clamp(min=1).double()[seq])
    else:
        per[:] = 1.0 / max(1, int(n.sum())) if case["agg"] == "token" else 1.0
    A = adv
    if case["per_seq"]:
        A = torch.zeros(T, device=DEV, dtype=torch.float64)
        A[first:first + len(seq)] = adv[seq]
    ratio = torch.exp(logp - old)
    unclipped, bounded = ratio * A, ratio.clamp(1 - 0.2, 1 + 0.28) * A
    hit = bounded < unclipped
    pol = -torch.minimum(unclipped, bounded)
    grad = torch.where(hit, 0.0, -unclipped)
    kl = torch.zeros_like(pol)
    if ref is not None:
        q = torch.exp(ref - logp)
        kl = q - 1 - (ref - logp)
        grad = grad + case["beta"] * (1 - q)
    w = per * ok
    tok = (pol + case["beta"] * kl) * ok
    return {"loss": (tok * w).sum().reshape(1), "tok_loss": tok,
            "diag": torch.stack([(pol * w).sum(1), (kl * w).sum(1), (hit * w).sum(1)]), "dlogp": grad * w}


def _exact_clip(case, seed):
    flat, views, most = _clip_inputs(case, seed)
    total = sum(float((b.double() ** 2).sum()) for b in flat.values())
    norm = math.sqrt(total)
    coef = 1.0 if math.isinf(most) else min(1.0, most / (norm + CLIP_EPS))
    return {"stats": torch.tensor([norm, coef], dtype=torch.float64),
            "grads": {k: b.double().mul_(coef) for k, b in flat.items()}}
