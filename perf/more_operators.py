"""Speculative decoding with a suite's shared key/value cache: the operators around the verify
step, each in a plain form and through the package.

  attn    attention of new tokens over a paged cache: the drafted tokens of a tree, a chain
          (prompts), or single tokens; every head of a group of query heads shares keys and values
  verify  acceptance of a drafted tree's tokens against the target's probabilities from given
          random numbers: the accepted path and the token that follows it
  round   the cache's pages over one decoding round: drop the last round's samples, fork new ones
          from their prompts, reserve, append the drafted tokens, keep the accepted path

A case is a dict of plain values.  ``listed`` gives fixed ones, ``draw`` more of the same
ranges.  Where ``own`` is false everything is computed with elementary torch operations.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
UNUSED = -2  # parent of a node that takes no part


def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


# ------------------------------------------------------------------------- cases
def listed():
    def attn(name, S, n, len, q_heads, kv_heads, dim, page, kind_of="tree", dtype="bf16", unused=0.0):
        return dict(name=name, kind="attn", S=S, n=n, len=len, q_heads=q_heads, kv_heads=kv_heads, dim=dim,
                    page=page, form=kind_of, dtype=dtype, unused=unused)

    def verify(name, S, n, V, width, draft="iid", cut=0.0):
        return dict(name=name, kind="verify", S=S, n=n, V=V, width=width, draft=draft, cut=cut)

    def round_(name, S, n, len, layers, kv_heads, dim, page, dtype="bf16"):
        return dict(name=name, kind="round", S=S, n=n, len=len, layers=layers, kv_heads=kv_heads, dim=dim,
                    page=page, dtype=dtype)

    return [
        # One user's verify round of a small sub-model: latency of interactive decoding.
        attn("tree_one", 1, 8, 700, 16, 4, 64, 16),
        # The verify round of a batch that is served together, prompts and answers of all lengths.
        attn("tree_batch", 32, 16, 4000, 32, 8, 128, 16),
        # Wide trees, as drafting with several candidates a position makes them.
        attn("tree_wide", 16, 64, 8000, 32, 8, 128, 64),
        # Plain decoding of many users, one token each.
        attn("decode", 128, 1, 4000, 32, 8, 128, 32, kind_of="chain"),
        # A few very long contexts, some nodes of the batch's trees padding.
        attn("tree_long", 4, 24, 131072, 32, 8, 128, 64, unused=0.1),
        # A piece of a prompt read into the cache behind what is there.
        attn("prompt", 4, 2048, 4096, 32, 8, 128, 64, kind_of="chain"),
        # Nothing round, in fp32: odd heads and widths, small pages.
        attn("tree_fp32", 5, 11, 301, 6, 2, 72, 8, dtype="fp32"),
        # One user's chain of drafted tokens: latency.
        verify("verify_one", 1, 7, 32003, 1),
        # The chains of the benchmark's verify batch, nucleus-like rows.
        verify("verify_batch", 102, 7, 50304, 1, cut=1e-3),
        # Trees of a served batch at the largest suite's vocabulary, siblings drawn without repetition.
        verify("verify_trees", 64, 32, 128256, 3, draft="distinct"),
        # One user's samples of a small sub-model: latency and the number of launches.
        round_("round_small", 4, 8, 200, 6, 4, 64, 16),
        # A group of samples for many prompts, all layers of a suite.
        round_("round_batch", 64, 32, 500, 28, 8, 128, 16),
    ]


_MOST_KV = 4 * 131072 * 8 * 128 * 4       # bytes of tree_long
_MOST_FLOPS = 4 * 4 * 2048 * 32 * 6144 * 128
_MOST_SCORES = 4 * 32 * 2048 * 6144
_MOST_ROWS = 64 * 32 * 128256             # values of verify_trees' rows
_MOST_ROUND = 64 * 32 * 28 * 8 * 128      # values that round_batch appends


def _log_int(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "verify", "verify", "round"])
    if kind == "attn":
        while True:
            dtype = rng.choice(["bf16", "bf16", "bf16", "bf16", "fp32"])
            form = rng.choice(["tree", "tree", "chain"])
            kv, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16])
            dim = rng.choice([64, 128, 128, 8 * rng.randint(4, 16)])
            S, length = _log_int(rng, 1, 256), _log_int(rng, 1, 131072)
            n = _log_int(rng, 1, 256) if form == "tree" else rng.choice([1, 1, _log_int(rng, 1, 2048)])
            case = dict(kind=kind, S=S, n=n, len=length, q_heads=kv * group, kv_heads=kv, dim=dim,
                        page=rng.choice([8, 16, 16, 32, 64, 128]), form=form, dtype=dtype,
                        unused=rng.choice([0.0, 0.0, 0.15]) if form == "tree" else 0.0)
            elt = 4 if dtype == "fp32" else 2
            scores = S * kv * group * n * (length + n)
            if (2 * S * (length + n) * kv * dim * elt <= _MOST_KV and scores <= _MOST_SCORES
                    and 4 * scores * dim <= (2e10 if dtype == "fp32" else _MOST_FLOPS)):
                return case
    if kind == "verify":
        while True:
            S, n, V = _log_int(rng, 1, 256), _log_int(rng, 1, 64), _log_int(rng, 500, 256000)
            if S * n * V <= _MOST_ROWS:
                return dict(kind=kind, S=S, n=n, V=V, width=rng.choice([1, 2, 3, 4, 6]),
                            draft=rng.choice(["iid", "distinct", "fixed"]), cut=rng.choice([0.0, 1e-3, 0.05]))
    while True:
        S, n, layers = _log_int(rng, 1, 128), _log_int(rng, 1, 64), _log_int(rng, 1, 48)
        kv, dim = rng.choice([1, 2, 4, 8, 16]), rng.choice([64, 128, 8 * rng.randint(4, 16)])
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        length = _log_int(rng, 1, 1000)
        if (S * n * layers * kv * dim * (2 if dtype == "fp32" else 1) <= _MOST_ROUND
                and 2 * S * (length + n) * layers * kv * dim <= 4 * _MOST_ROUND * 8):
            return dict(kind=kind, S=S, n=n, len=length, layers=layers, kv_heads=kv, dim=dim,
                        page=rng.choice([8, 16, 32, 64]), dtype=dtype)


# ------------------------------------------------------------------------- inputs
def _gen(seed, k):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 8 + k)
    return g


def _lengths(case):
    """Per sequence what its cache holds and how many new tokens it has: ragged, but of the case alone."""
    rng = random.Random(case["S"] * 1000003 + case["len"] * 101 + case["n"])
    S, n, most = case["S"], case["n"], case["len"]
    lens = [most] + [int(most * rng.random()) if rng.random() < 0.7 else most - rng.randint(0, min(most, 63))
                     for _ in range(S - 1)]
    news = [n] + [n if rng.random() < 0.5 else rng.randint(max(1, n // 2), n) for _ in range(S - 1)]
    return lens, news


def _starts(news):
    at = [0]
    for n in news:
        at.append(at[-1] + n)
    return at


def _local(news):
    """Per packed node its sequence and its number within it, on the GPU."""
    n = torch.tensor(news, device=DEV)
    seq = torch.repeat_interleave(torch.arange(len(news), device=DEV), n)
    first = torch.cumsum(n, 0) - n
    return seq, torch.arange(sum(news), device=DEV) - first[seq]


def _attn_inputs(case, seed):
    """A cache whose pages lie in any order, queries that favour a few keys, trees whose nodes
    hang below one of the last few nodes."""
    lens, news = _lengths(case)
    S, page, kv, dim, dt, g = case["S"], case["page"], case["kv_heads"], case["dim"], _dtype(case), _gen(seed, 0)
    held = [-(-(a + b) // page) for a, b in zip(lens, news)]
    pages, most = sum(held) + 7, max(held)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.full((S, most), -1, dtype=torch.int32, device=DEV)
    at = _starts(held)
    col = torch.arange(most, device=DEV)
    h = torch.tensor(held, device=DEV)[:, None]
    table = torch.where(col < h, order[(torch.tensor(at[:-1], device=DEV)[:, None] + col).clamp(max=pages - 1)], table)
    k = torch.randn(1, pages, kv, page, dim, generator=g, device=DEV, dtype=dt)
    v = torch.randn(1, pages, kv, page, dim, generator=g, device=DEV, dtype=dt)
    N = sum(news)
    q = torch.randn(N, case["q_heads"], dim, generator=g, device=DEV).mul_(2.0).to(dt)
    _, i = _local(news)
    parents = None
    if case["form"] == "tree":
        back = (torch.rand(N, generator=g, device=DEV) * torch.minimum(i, torch.full_like(i, 4))).long()
        parents = i - 1 - back
        loose = torch.rand(N, generator=g, device=DEV) < case["unused"]
        parents = torch.where(loose & (i > 0), UNUSED, parents).to(torch.int32)
    start = torch.tensor(_starts(news), dtype=torch.int32, device=DEV)
    return dict(k=k, v=v, table=table, lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
                held=torch.tensor(held, dtype=torch.int32, device=DEV), q=q, parents=parents, start=start)


def _verify_inputs(case, seed):
    """Draft and target rows whose logits share most of their spread, the tokens drawn from the
    draft's rows (or its most likely ones, where the draft gives no probabilities)."""
    S, n, V, w = case["S"], case["n"], case["V"], case["width"]
    g = _gen(seed, 0)
    _, news = _lengths(dict(S=S, n=n, len=V))
    N = sum(news)
    _, i = _local(news)
    back = (torch.rand(N, generator=g, device=DEV) * torch.minimum(i, torch.full_like(i, w))).long()
    parents = (i - 1 - back).to(torch.int32)
    p = torch.empty(N, V, device=DEV)
    q = torch.empty(N, V, device=DEV)
    top = torch.empty(N, w, dtype=torch.int64, device=DEV)
    step = max(1, (1 << 27) // V)
    for a in range(0, N, step):
        m = min(step, N - a)
        z = torch.randn(m, V, generator=g, device=DEV).mul_(2.5)
        zt = z + torch.randn(m, V, generator=g, device=DEV).mul_(0.7)
        for rows, logits in ((q, z), (p, zt)):
            e = torch.exp((logits - logits.max(1, keepdim=True).values) / 0.7)
            e = torch.where(e < case["cut"], 0.0, e)
            rows[a:a + m] = e / e.sum(1, keepdim=True)
        if case["draft"] == "fixed":
            score = q[a:a + m]
        else:
            score = torch.log(q[a:a + m]) - torch.log(-torch.log(torch.rand(m, V, generator=g, device=DEV).clamp_(1e-9, 0.9999999)))
        many = torch.topk(score, w, dim=1).indices
        if case["draft"] == "iid":  # one winner of a noise of its own for each sibling
            for c in range(1, w):
                noise = torch.log(-torch.log(torch.rand(m, V, generator=g, device=DEV).clamp_(1e-9, 0.9999999)))
                many[:, c] = (torch.log(q[a:a + m]) - noise).argmax(1)
        top[a:a + m] = many
    # a node's number among its siblings picks its token
    start = torch.tensor(_starts(news), device=DEV)
    seq, _ = _local(news)
    up = start[seq] + parents.long()
    rank = torch.zeros(N, dtype=torch.int64, device=DEV)
    for b in range(1, w):  # siblings lie within w nodes
        same = torch.zeros(N, dtype=torch.bool, device=DEV)
        same[b:] = (up[b:] == up[:-b]) & (parents[b:] >= 0) & (seq[b:] == seq[:-b])
        rank += same
    tokens = torch.where(parents >= 0, top[up.clamp(min=0), rank.clamp(max=w - 1)], 0).to(torch.int32)
    u = torch.rand(N, 2, generator=g, device=DEV)
    return dict(p=p, q=None if case["draft"] == "fixed" else q, tokens=tokens, parents=parents,
                start=start.to(torch.int32), u=u)


def _round_sizes(case):
    lens, news = _lengths(case)
    page = case["page"]
    most = -(-(case["len"] + case["n"]) // page)
    pages = sum(-(-a // page) for a in lens) + sum(-(-b // page) + 2 for b in news) + 5
    return lens, news, pages, most


def _round_inputs(case, seed):
    """The prompts' pages as they were reserved one after the other, whatever an earlier use left
    in the pool, new keys and values for the drafted tokens, and the paths that verification kept."""
    lens, news, pages, most = _round_sizes(case)
    S, page, kv, dim, L, dt, g = (case["S"], case["page"], case["kv_heads"], case["dim"], case["layers"],
                                  _dtype(case), _gen(seed, 0))
    k = torch.randn(L, pages, kv, page, dim, generator=g, device=DEV, dtype=dt)
    v = torch.randn(L, pages, kv, page, dim, generator=g, device=DEV, dtype=dt)
    N = sum(news)
    kn = torch.randn(L, N, kv, dim, generator=g, device=DEV, dtype=dt)
    vn = torch.randn(L, N, kv, dim, generator=g, device=DEV, dtype=dt)
    n = torch.tensor(news, device=DEV)
    step = torch.randint(1, 4, (S, case["n"]), generator=g, device=DEV)
    step[:, 0] = 0
    path = step.cumsum(1)
    inside = (path < n[:, None]).sum(1)
    keep = torch.minimum(inside, 1 + (torch.rand(S, generator=g, device=DEV) * 6).long())
    path = torch.where(torch.arange(case["n"], device=DEV) < keep[:, None], path, -1).to(torch.int32)
    return dict(k=k, v=v, kn=kn, vn=vn, path=path, keep=keep.to(torch.int32),
                lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
                news=n.to(torch.int32), start=torch.tensor(_starts(news), dtype=torch.int32, device=DEV))


def _round_start(case, inp):
    """The cache's state with the prompts in it: rows 0 .. S-1, pages from the lowest on."""
    lens, _, pages, most = _round_sizes(case)
    S, page = case["S"], case["page"]
    held = torch.tensor([-(-a // page) for a in lens], device=DEV)
    first = torch.cumsum(held, 0) - held
    col = torch.arange(most, device=DEV)
    table = torch.full((2 * S, most), -1, dtype=torch.int32, device=DEV)
    table[:S] = torch.where(col < held[:, None], first[:, None] + col, -1).to(torch.int32)
    zero = torch.zeros(S, dtype=torch.int32, device=DEV)
    refs = (torch.arange(pages, device=DEV) < held.sum()).to(torch.int32)
    return dict(table=table, len=torch.cat([inp["lens"], zero]), held=torch.cat([held.to(torch.int32), zero]), refs=refs)


# ------------------------------------------------------------------------- passes
def prepare(case, seed):
    kind = case["kind"]
    s = {"case": case, "kind": kind}
    s["in"] = inp = {"attn": _attn_inputs, "verify": _verify_inputs, "round": _round_inputs}[kind](case, seed)
    S = case["S"]
    if kind == "round":
        s["state"] = _round_start(case, inp)
        s["parent"] = torch.arange(S, dtype=torch.int32, device=DEV)
        s["child"] = s["parent"] + S
    if own:  # the cache and the handles with their outputs and workspace, kept from step to step
        import paper_2608_09703_gb300 as mls

        if kind == "verify":
            s["op"] = mls.TreeVerify(S, inp["tokens"].numel(), case["V"], max_path=case["n"],
                                     replace=case["draft"] != "distinct", device=DEV)
            return s
        k = inp.pop("k")
        table = inp["table"] if kind == "attn" else s["state"]["table"]
        c = s["cache"] = mls.PagedCache(k.shape[0], k.shape[1], case["page"], case["kv_heads"], case["dim"],
                                        seqs=table.shape[0], max_pages=table.shape[1], dtype=k.dtype, device=DEV)
        c.k.copy_(k)
        c.v.copy_(inp.pop("v"))
        if kind == "attn":
            c.table.copy_(table)
            c.len.copy_(inp["lens"])
            c.held.copy_(inp["held"])
            s["op"] = mls.TreeAttention(c, S, inp["q"].shape[0], case["q_heads"])
        else:  # the prompts
            c.reserve(inp["lens"], seqs=s["parent"])
            c.compact(inp["lens"], seqs=s["parent"])
    return s


def run(s):
    if own:
        return _run_own(s)
    return {"attn": _plain_attn, "verify": _plain_verify, "round": _plain_round}[s["kind"]](s)


def _run_own(s):
    kind, i = s["kind"], s["in"]
    if kind == "attn":
        out, lse = s["op"](i["q"], i["start"], parents=i["parents"])
        return {"out": out, "lse": lse}
    if kind == "verify":
        n_path, path, token = s["op"](i["p"], i["tokens"], i["parents"], i["start"], i["u"], draft=i["q"])
        return {"n_path": n_path, "path": path, "next_token": token}
    c = s["cache"]
    c.free(s["child"])
    c.fork(s["parent"], s["child"])
    c.reserve(i["news"], seqs=s["child"])
    c.append(i["kn"], i["vn"], i["start"], seqs=s["child"])
    c.compact(i["keep"], path=i["path"], seqs=s["child"])
    return {"k": c.k, "v": c.v, "table": c.table, "len": c.len, "held": c.held, "refs": c.refs}


def _visible(case, parents, start, lens, n, L):
    """[S, n, L]: which positions of the cache each new token attends to."""
    S = len(lens)
    i = torch.arange(n, device=DEV)
    real = i < (start[1:] - start[:-1])[:, None]
    if parents is None:
        below = torch.tril(torch.ones(n, n, device=DEV, dtype=torch.bool)).expand(S, n, n)
        used = real
    else:
        p = torch.full((S, n), UNUSED, dtype=torch.int64, device=DEV)
        p[real] = parents.long()
        used = real & (p >= -1)
        edge = (p[:, :, None] == i) & used[:, :, None] & used[:, None, :]
        reach = (edge | torch.eye(n, device=DEV, dtype=torch.bool)).float()
        for _ in range(max(1, math.ceil(math.log2(n)))):  # paths of twice the length each time
            reach = (reach @ reach > 0).float()
        below = reach > 0
    at = torch.arange(L, device=DEV) - lens.long()[:, None]
    at = at[:, None, :].expand(S, n, L)
    tree = torch.gather(below & used[:, :, None], 2, at.clamp(0, n - 1))
    return torch.where(at < 0, used[:, :, None], tree & (at < n)), real


def _plain_attn(s):
    case, x = s["case"], s["in"]
    S, n, kv, D, page = case["S"], case["n"], case["kv_heads"], case["dim"], case["page"]
    G = case["q_heads"] // kv
    pages = x["table"].clamp(min=0).long()
    L = pages.shape[1] * page
    see, real = _visible(case, x["parents"], x["start"], x["lens"], n, L)
    K = x["k"][0][pages].permute(0, 2, 1, 3, 4).reshape(S, kv, L, D).float()
    Q = torch.zeros(S, n, kv, G, D, device=DEV)
    Q[real] = x["q"].float().view(-1, kv, G, D)
    z = (Q.permute(0, 2, 1, 3, 4).reshape(S, kv, n * G, D) @ K.transpose(2, 3)).mul_(D ** -0.5)
    del K
    z = z.view(S, kv, n, G, L).masked_fill_(~see[:, None, :, None, :], -math.inf)
    top = z.amax(4, keepdim=True)
    floor = torch.where(top == -math.inf, 0.0, top)
    e = z.sub_(floor).exp_()
    total = e.sum(4, keepdim=True)
    lse = (floor + torch.log(total))[..., 0]
    e.div_(torch.where(total == 0, 1.0, total))
    V = x["v"][0][pages].permute(0, 2, 1, 3, 4).reshape(S, kv, L, D).float()
    out = (e.view(S, kv, n * G, L) @ V).view(S, kv, n, G, D).permute(0, 2, 1, 3, 4)
    return {"out": out[real].reshape(-1, kv * G, D).to(x["q"].dtype),
            "lse": lse.permute(0, 2, 1, 3)[real].reshape(-1, kv * G)}


def _plain_verify(s):
    """All sequences at once, node after node; the residual as its definition has it."""
    case, x = s["case"], s["in"]
    S, n, V = case["S"], case["n"], case["V"]
    start, tokens, parents, u = x["start"].long(), x["tokens"].long(), x["parents"].long(), x["u"].double()
    news = start[1:] - start[:-1]
    cur = torch.zeros(S, dtype=torch.int64, device=DEV)
    path = torch.full((S, n), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = 0
    count = torch.ones(S, dtype=torch.int64, device=DEV)
    R = x["p"][start[:-1]].double()
    Q = None if x["q"] is None else x["q"][start[:-1]].double()
    rows = torch.arange(S, device=DEV)
    for c in range(1, n):
        node = (start[:-1] + c).clamp(max=len(tokens) - 1)
        child = (c < news) & (parents[node] == cur)
        t = tokens[node]
        fits = (t >= 0) & (t < V)
        t = t.clamp(0, V - 1)
        q = torch.ones(S, dtype=torch.float64, device=DEV) if Q is None else Q[rows, t]
        ok = child & fits & (q > 0) & (u[node, 0] * q < R[rows, t])
        no = child & ~ok
        if Q is None:
            left = R.clone()
            left[rows, t] = torch.where(fits, 0.0, left[rows, t])
        else:
            left = (R - Q).clamp_(min=0)
        mass = left.sum(1)
        change = no & (mass > 0)
        R = torch.where(change[:, None], left / mass.clamp(min=1e-300)[:, None], R)
        if Q is not None and case["draft"] == "distinct":
            less = Q.clone()
            less[rows, t] = torch.where(fits, 0.0, less[rows, t])
            mass = less.sum(1)
            Q = torch.where((no & (mass > 0))[:, None], less / mass.clamp(min=1e-300)[:, None],
                            torch.where(no[:, None], 0.0, Q))
        R = torch.where(ok[:, None], x["p"][node].double(), R)
        if Q is not None:
            Q = torch.where(ok[:, None], x["q"][node].double(), Q)
        cur = torch.where(ok, c, cur)
        path = torch.where(ok[:, None] & (torch.arange(n, device=DEV) == count[:, None]), c, path)
        count = count + ok
    cum = R.cumsum(1)
    goal = u[start[:-1] + cur, 1] * cum[:, -1]
    token = torch.searchsorted(cum, goal[:, None], right=True)[:, 0]
    return {"n_path": count.to(torch.int32), "path": path.to(torch.int32), "next_token": token.to(torch.int32)}


def _plain_take(state, rows, first, count):
    """Gives each of `rows` the lowest free pages for its columns first .. first + count."""
    refs, table = state["refs"], state["table"]
    number = torch.arange(len(refs), device=DEV)
    free = torch.sort(torch.where(refs == 0, number, number + len(refs))).indices
    upto = count.cumsum(0)
    col = torch.arange(table.shape[1], device=DEV)
    mine = (col >= first[:, None]) & (col < (first + count)[:, None])
    which = ((upto - count)[:, None] + col - first[:, None]).clamp(0, len(free) - 1)
    table[rows] = torch.where(mine, free[which].to(torch.int32), table[rows])
    refs[free] = torch.where((number < upto[-1]), 1, refs[free])


def _plain_drop(state, rows, keep):
    """Gives back the pages of `rows` from column `keep` on."""
    table, held, refs = state["table"], state["held"], state["refs"]
    col = torch.arange(table.shape[1], device=DEV)
    gone = (col >= keep[:, None]) & (col < held[rows][:, None])
    refs.index_add_(0, table[rows].clamp(min=0).long().reshape(-1), -gone.to(torch.int32).reshape(-1))
    table[rows] = torch.where(gone, -1, table[rows])
    held[rows] = keep.to(torch.int32)


def _plain_round(s):
    case, x, st = s["case"], s["in"], s["state"]
    page, parent, child = case["page"], s["parent"].long(), s["child"].long()
    k, v, table, length, held, refs = x["k"], x["v"], st["table"], st["len"], st["held"], st["refs"]
    zero = torch.zeros_like(child)
    # free
    _plain_drop(st, child, zero)
    length[child] = 0
    # fork: full pages shared, the last one copied where it is partly filled
    n = length[parent].long()
    full = n // page
    part = (n % page > 0).long()
    col = torch.arange(table.shape[1], device=DEV)
    shared = col < full[:, None]
    table[child] = torch.where(shared, table[parent], -1)
    refs.index_add_(0, table[parent].clamp(min=0).long().reshape(-1), shared.to(torch.int32).reshape(-1))
    _plain_take(st, child, full, part)
    last = (full - 1 + part).clamp(min=0)[:, None]
    src, dst = (table[r].gather(1, last)[:, 0].clamp(min=0).long() for r in (parent, child))
    slot = torch.arange(page, device=DEV)
    fill = ((slot < (n % page)[:, None]) & (part > 0)[:, None])[None, :, None, :, None]
    for pool in (k, v):
        pool[:, dst] = torch.where(fill, pool[:, src], pool[:, dst])
    length[child] = n.to(torch.int32)
    held[child] = (full + part).to(torch.int32)
    # reserve
    have = held[child].long()
    need = (n + x["news"] + page - 1) // page - have
    _plain_take(st, child, have, need)
    held[child] = (have + need).to(torch.int32)
    # append
    seq = torch.repeat_interleave(torch.arange(len(child), device=DEV), x["news"].long(), output_size=x["kn"].shape[1])
    at = n[seq] + torch.arange(len(seq), device=DEV) - x["start"].long()[seq]
    where = table[child][seq, at // page].long()
    k[:, where, :, at % page] = x["kn"].permute(1, 0, 2, 3)
    v[:, where, :, at % page] = x["vn"].permute(1, 0, 2, 3)
    # compact: the kept path's tokens side by side (a place that keeps nothing writes its first again)
    path = x["path"].long()
    j = torch.arange(path.shape[1], device=DEV)
    kept = j < x["keep"][:, None]
    a = n[:, None] + torch.where(kept, path, 0)
    b = n[:, None] + torch.where(kept, j, 0)
    pa, pb = (table[child].gather(1, t // page).long().reshape(-1) for t in (a, b))
    for pool in (k, v):
        pool[:, pb, :, (b % page).reshape(-1)] = pool[:, pa, :, (a % page).reshape(-1)]
    length[child] += x["keep"]
    _plain_drop(st, child, (length[child].long() + page - 1) // page)
    return {"k": k, "v": v, "table": table, "len": length, "held": held, "refs": refs}


def work(case):
    """Each input read once, each output written once, and the products that the definitions need."""
    kind = case["kind"]
    if kind == "verify":  # the draft's and the target's row where each walk ends, and the nodes
        _, news = _lengths(dict(S=case["S"], n=case["n"], len=case["V"]))
        rows = 1 if case["draft"] == "fixed" else 2
        return {"bytes": 4 * case["S"] * case["V"] * rows + sum(news) * 24 + case["S"] * (4 * case["n"] + 12),
                "flops": case["S"] * case["V"] * 2 * rows}
    lens, news = _lengths(case)
    elt = 4 if case["dtype"] == "fp32" else 2
    D, kv = case["dim"], case["kv_heads"]
    if kind == "attn":
        N, Hq = sum(news), case["q_heads"]
        pairs = sum(n * (a + (n + 1) / 2) if case["form"] == "chain" else n * (a + min(n, 8)) for a, n in zip(lens, news))
        return {"bytes": 2 * sum(a + n for a, n in zip(lens, news)) * kv * D * elt + 2 * N * Hq * D * elt + 4 * N * Hq
                + 4 * sum(-(-(a + n) // case["page"]) for a, n in zip(lens, news)) + 8 * case["S"] + 4 * N,
                "flops": 4 * Hq * D * pairs}
    token = 2 * case["layers"] * kv * D * elt  # a token's keys and values
    copied = sum(a % case["page"] for a in lens)
    return {"bytes": 2 * token * (copied + sum(news) + 2 * case["S"]) + 16 * sum(news), "flops": 0}


# ------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    return {"attn": _exact_attn, "verify": _exact_verify, "round": _exact_round}[case["kind"]](case, seed)


def _exact_attn(case, seed):
    """Sequence by sequence, its tokens put in order first; each node's path walked on the host."""
    lens, news = _lengths(case)
    x = _attn_inputs(case, seed)
    kv, D, page = case["kv_heads"], case["dim"], case["page"]
    G = case["q_heads"] // kv
    up = None if x["parents"] is None else x["parents"].tolist()
    outs, lses, at = [], [], 0
    for b, (have, n) in enumerate(zip(lens, news)):
        total = have + n
        pages = x["table"][b, :-(-total // page)].long()
        K = x["k"][0, pages].transpose(1, 2).reshape(-1, kv, D)[:total]
        V = x["v"][0, pages].transpose(1, 2).reshape(-1, kv, D)[:total]
        see = torch.zeros(n, n, dtype=torch.bool)
        for i in range(n):
            if up is None:
                see[i, :i + 1] = True
                continue
            j = i
            while j >= 0 and up[at + j] >= -1:
                see[i, j] = True
                j = up[at + j]
        see = see.to(DEV)
        alive = see.any(1)
        for h in range(kv):
            Kh, Vh = K[:, h].double(), V[:, h].double()
            o = torch.empty(n, G, D, dtype=torch.float64, device=DEV)
            ls = torch.empty(n, G, dtype=torch.float64, device=DEV)
            step = max(1, (1 << 27) // (G * total))
            for a in range(0, n, step):
                qh = x["q"][at + a:at + min(n, a + step), h * G:(h + 1) * G].double()
                z = torch.einsum("ngd,td->ngt", qh, Kh) / math.sqrt(D)
                m = torch.cat([alive[a:a + step, None].expand(-1, have), see[a:a + step]], 1)
                z = torch.where(m[:, None], z, -math.inf)
                l = torch.logsumexp(z, 2)
                ls[a:a + step] = l
                o[a:a + step] = torch.where(alive[a:a + step, None, None],
                                            torch.einsum("ngt,td->ngd", torch.exp(z - torch.where(l == -math.inf, 0.0, l)[..., None]), Vh), 0.0)
            outs.append(o)
            lses.append(ls)
        at += n
    out = torch.cat([torch.cat(outs[b * kv:(b + 1) * kv], 1) for b in range(len(lens))])
    lse = torch.cat([torch.cat(lses[b * kv:(b + 1) * kv], 1) for b in range(len(lens))])
    return {"out": out, "lse": lse}


def _exact_verify(case, seed):
    """One sequence after the other: a residual after j refusals is max(0, p - c q) over its sum,
    where c adds up what the refusals before it left."""
    x = _verify_inputs(case, seed)
    start, tokens, parents, u = (x[k].tolist() for k in ("start", "tokens", "parents", "u"))
    _, news = _lengths(dict(S=case["S"], n=case["n"], len=case["V"]))
    paths, ends = [], []
    for b, n in enumerate(news):
        at, path, c = start[b], [0], 0
        while True:
            p = x["p"][at + c].double()
            q = None if x["q"] is None else x["q"][at + c].double()
            w, mass, gone, share, nxt = p, 1.0, torch.zeros_like(p), 1.0, None
            take = torch.zeros_like(p)  # how much of the draft's row has been taken off each token
            for d in range(c + 1, n):
                if parents[at + d] != c:
                    continue
                t = tokens[at + d]
                if q is None:
                    if u[at + d][0] < float(w[t]) / mass:
                        nxt = d
                        break
                    new = w.clone()
                    new[t] = 0.0
                    if float(new.sum()) > 0:
                        w, mass = new, float(new.sum())
                    continue
                qt = 0.0 if gone[t] > 0 and case["draft"] == "distinct" else float(q[t]) * share
                if qt > 0 and u[at + d][0] * qt < float(w[t]) / mass:
                    nxt = d
                    break
                live = torch.where(gone > 0, 0.0, q) if case["draft"] == "distinct" else q
                new = (p - take - live * (share * mass)).clamp_(min=0)
                if float(new.sum()) > 0:
                    take = take + live * (share * mass)
                    w, mass = new, float(new.sum())
                if case["draft"] == "distinct":
                    gone[t] = 1.0
                    left = float(torch.where(gone > 0, 0.0, q).sum())
                    share = 1.0 / left if left > 0 else 0.0
            if nxt is None:
                cum = w.cumsum(0)
                ends.append(int((cum <= u[at + c][1] * cum[-1]).sum()))
                break
            path.append(nxt)
            c = nxt
        paths.append(path)
    rows = torch.full((case["S"], case["n"]), -1, dtype=torch.int32)
    for b, path in enumerate(paths):
        rows[b, :len(path)] = torch.tensor(path, dtype=torch.int32)
    return {"n_path": torch.tensor([len(r) for r in paths], dtype=torch.int32).to(DEV), "path": rows.to(DEV),
            "next_token": torch.tensor(ends, dtype=torch.int32).to(DEV)}


def _exact_round(case, seed):
    """The pages handed out and taken back one by one, each token moved by itself (whole numbers and copies)."""
    x = _round_inputs(case, seed)
    lens, news, pages, most = _round_sizes(case)
    S, page, L = case["S"], case["page"], case["layers"]
    refs, rows, length, nextp = [0] * pages, [], list(lens) + [0] * S, 0
    for a in lens:
        rows.append(list(range(nextp, nextp + -(-a // page))))
        for r in rows[-1]:
            refs[r] = 1
        nextp += -(-a // page)
    free = [r for r in range(pages) if refs[r] == 0][::-1]

    def take():
        refs[free[-1]] = 1
        return free.pop()

    k, v = x["k"].clone(), x["v"].clone()
    for b in range(S):
        row = rows[b][:lens[b] // page]
        for r in row:
            refs[r] += 1
        if lens[b] % page:
            new, old, m = take(), rows[b][-1], lens[b] % page
            k[:, new, :, :m] = k[:, old, :, :m]
            v[:, new, :, :m] = v[:, old, :, :m]
            row = row + [new]
        rows.append(row)
    for b in range(S):
        while len(rows[S + b]) * page < lens[b] + news[b]:
            rows[S + b].append(take())
    paths, keep, at = x["path"].tolist(), x["keep"].tolist(), 0
    for b in range(S):
        row, n = torch.tensor(rows[S + b], device=DEV), lens[b]
        pos = torch.arange(n, n + news[b], device=DEV)
        kept = torch.tensor([n + j for j in paths[b][:keep[b]]], device=DEV)
        to = torch.arange(n, n + keep[b], device=DEV)
        for pool, fresh in ((k, x["kn"]), (v, x["vn"])):
            pool[:, row[pos // page], :, pos % page] = fresh[:, at:at + news[b]].transpose(0, 1)
            pool[:, row[to // page], :, to % page] = pool[:, row[kept // page], :, kept % page]
        at += news[b]
        length[S + b] = n + keep[b]
        for r in rows[S + b][-(-length[S + b] // page):]:
            refs[r] -= 1
        rows[S + b] = rows[S + b][:-(-length[S + b] // page)]
    table = torch.tensor([r + [-1] * (most - len(r)) for r in rows], dtype=torch.int32, device=DEV)
    return {"k": k, "v": v, "table": table, "len": torch.tensor(length, dtype=torch.int32, device=DEV),
            "held": torch.tensor([len(r) for r in rows], dtype=torch.int32, device=DEV),
            "refs": torch.tensor(refs, dtype=torch.int32, device=DEV)}
