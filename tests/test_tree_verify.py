"""Acceptance of drafted trees against the definition in 64 bits, node after node: every decision and the
token drawn have to be equal.  A decision that the exact values leave within 1e-9 of a border (of the whole's
share) could go either way by rounding in 64 bits itself; the few sequences with one are left out, by the
definition's own values and not by the kernel's answer."""
import numpy as np
import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B

NEAR = 1e-9


def walk(p, q, tokens, parents, u, mode):
    """(path, next token, nearest border) of one sequence, in 64 bits.  mode: iid, distinct or fixed."""
    n, V = p.shape
    cur, path, near = 0, [0], np.inf
    while True:
        r, rest = p[cur].astype(np.float64), None if q is None else q[cur].astype(np.float64)
        taken = None
        for d in range(cur + 1, n):
            if parents[d] != cur:
                continue
            x = int(tokens[d])
            inside = 0 <= x < V
            qx = 1.0 if q is None else (rest[x] if inside else 0.0)
            if inside and qx > 0:
                near = min(near, abs(float(u[d, 0]) * qx - r[x]) / max(qx, r[x]) if max(qx, r[x]) > 0 else np.inf)
                if float(u[d, 0]) * qx < r[x]:
                    taken = d
                    break
            if q is None:
                left = r.copy()
                if inside:
                    left[x] = 0.0
            else:
                left = np.maximum(0.0, r - rest)
            if left.sum() > 0:
                r = left / left.sum()
            if mode == "distinct":
                if inside:
                    rest = rest.copy()
                    rest[x] = 0.0
                rest = rest / rest.sum() if rest.sum() > 0 else rest * 0.0
        if taken is None:
            cum = np.cumsum(r)
            if not cum[-1] > 0:
                return path, -1, near
            goal = float(u[cur, 1]) * cum[-1]
            at = int(np.searchsorted(cum, goal, side="right"))
            if goal > 0:
                near = min(near, np.abs(cum - goal).min() / cum[-1])
            return path, at, near
        path.append(taken)
        cur = taken


def make(S, n, V, width, seed, mode, flat=1.0, cut=0.0, device="cpu", ragged=True):
    g = torch.Generator().manual_seed(seed)
    news = [int(torch.randint(0 if ragged else n, n + 1, (1,), generator=g)) for _ in range(S)]
    if ragged and S > 1:
        news[0], news[1] = 0, n
    start = np.concatenate([[0], np.cumsum(news)])
    N = int(start[-1])
    z = torch.randn(N, V, generator=g) * 2.0 * flat
    zt = z + torch.randn(N, V, generator=g) * 0.8

    def rows(logits):
        e = torch.exp(logits.double() - logits.double().max(1, keepdim=True).values if N else logits.double())
        e = torch.where(e < cut, 0.0, e)
        return (e / e.sum(1, keepdim=True)).float()

    p, q = rows(zt), rows(z)
    parents, tokens = np.full(N, -1, np.int32), np.zeros(N, np.int32)
    used = {}
    rng = np.random.RandomState(seed + 1)
    for b in range(S):
        for i in range(1, news[b]):
            up = i - 1 - rng.randint(0, min(i, width))
            parents[start[b] + i] = up
            row = q[start[b] + up].double().numpy()
            row = row / row.sum()
            key = (b, up)
            if mode == "distinct":
                for x in used.get(key, []):
                    row[x] = 0.0
            if mode == "fixed":
                order = np.argsort(-row)
                x = int(order[len(used.get(key, [])) % V])
            else:
                x = int(rng.choice(V, p=row / row.sum())) if row.sum() > 0 else 0
            used.setdefault(key, []).append(x)
            tokens[start[b] + i] = x
    u = torch.rand(N, 2, generator=g)
    return dict(p=p, q=None if mode == "fixed" else q, tokens=torch.from_numpy(tokens), parents=torch.from_numpy(parents),
                start=torch.from_numpy(start.astype(np.int32)), u=u, news=news, V=V, mode=mode, n=n)


def expected(x):
    out = []
    for b in range(len(x["news"])):
        a, e = int(x["start"][b]), int(x["start"][b + 1])
        if a == e:
            out.append(([], -1, np.inf))
            continue
        out.append(walk(x["p"][a:e].numpy(), None if x["q"] is None else x["q"][a:e].numpy(), x["tokens"][a:e].numpy(),
                        x["parents"][a:e].numpy(), x["u"][a:e].numpy(), x["mode"]))
    return out


def run(x, max_path=None, device="cuda"):
    def d(t):
        return None if t is None else t.to(device)

    op = mls.TreeVerify(len(x["news"]), x["p"].shape[0], x["V"], max_path=max_path or max(x["n"], 1),
                        replace=x["mode"] != "distinct")
    got = op(d(x["p"]), d(x["tokens"]), d(x["parents"]), d(x["start"]), d(x["u"]), draft=d(x["q"]))
    return [t.cpu().numpy() for t in got]


def check(x, got, least=0.98):
    n_path, path, token = got
    sure = 0
    for b, (want, nxt, near) in enumerate(expected(x)):
        if near < NEAR:
            continue
        sure += 1
        assert n_path[b] == len(want), (b, path[b], want)
        assert path[b, :len(want)].tolist() == want and (path[b, len(want):] == -1).all(), (b, path[b], want)
        assert token[b] == nxt, (b, token[b], nxt)
    assert sure >= least * len(x["news"])


# one sequence (a cluster of CTAs), a cluster of two, one CTA each; rows shorter than a warp's span, of one value,
# not a multiple of anything; chains and bushy trees
CASES = [(1, 7, 50304, 1), (1, 1, 9000, 1), (3, 12, 33001, 3), (60, 9, 9001, 2), (200, 6, 517, 4), (170, 5, 31, 6),
         (5, 4, 1, 2), (4, 256, 40, 5), (2, 256, 700, 200)]


@pytest.mark.gpu
@pytest.mark.parametrize("mode", ["iid", "distinct", "fixed"])
@pytest.mark.parametrize("S,n,V,width", CASES)
def test_against_the_definition(S, n, V, width, mode):
    x = make(S, n, V, width, seed=S + n + V, mode=mode)
    check(x, run(x))
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("mode", ["iid", "distinct", "fixed"])
@pytest.mark.parametrize("flat,cut", [(0.01, 0.0), (4.0, 0.02), (8.0, 0.5)])
def test_flat_and_peaked_rows(mode, flat, cut):
    x = make(40, 10, 5003, 4, seed=17, mode=mode, flat=flat, cut=cut)
    check(x, run(x))


@pytest.mark.gpu
def test_equal_rows_accept_all_and_refusals_without_rest():
    """p = q: every drawn child is accepted where it is drawn first; a second one too, for nothing is
    ever refused.  u = 1 - 2^-24 against p slightly below q refuses where p <= q everywhere: r stays."""
    x = make(50, 8, 300, 3, seed=5, mode="iid", ragged=False)
    x["p"] = x["q"].clone()
    n_path, path, _ = run(x)
    for b in range(50):
        a, cur, want = int(x["start"][b]), 0, [0]
        while True:
            kids = [d for d in range(cur + 1, 8) if int(x["parents"][a + d]) == cur]
            if not kids:
                break
            cur = kids[0]
            want.append(cur)
        assert path[b, :n_path[b]].tolist() == want
    for mode in ("iid", "distinct"):
        y = make(50, 8, 300, 3, seed=6, mode=mode, ragged=False)
        y["p"] = y["q"] * 0.5
        y["u"][:, 0] = 0.75
        check(y, run(y))


@pytest.mark.gpu
def test_tokens_outside_repeated_siblings_and_zero_draws():
    for mode in ("iid", "distinct", "fixed"):
        x = make(64, 12, 1000, 6, seed=9, mode=mode, ragged=False)
        x["tokens"][1::5] = -1
        x["tokens"][2::7] = 1000
        x["tokens"][3::6] = x["tokens"][4::6].clone()  # 64 x 12 nodes: as many of each
        x["u"][::3, 1] = 0.0
        x["u"][1::4, 0] = 0.0
        check(x, run(x), least=0.9)
        assert mls.mls_get_status() == 0


@pytest.mark.gpu
def test_distribution_of_the_first_token():
    """The point of it all: whatever was drafted, the first token emitted is distributed as p.  20000
    sequences of three children each; 4.5 sigma of each token's count."""
    S, V = 20000, 6
    g = torch.Generator().manual_seed(3)
    p = torch.tensor([0.05, 0.3, 0.2, 0.05, 0.1, 0.3])
    q = torch.tensor([0.4, 0.1, 0.1, 0.2, 0.1, 0.1])
    for mode in ("iid", "distinct", "fixed"):
        tokens = torch.zeros(S, 4, dtype=torch.int32)
        if mode == "fixed":
            tokens[:, 1:] = torch.tensor([5, 1, 0], dtype=torch.int32)
        else:
            tokens[:, 1:] = torch.multinomial(q.expand(S, V), 3, replacement=mode == "iid", generator=g).int()
        x = dict(p=p.repeat(4 * S, 1), q=None if mode == "fixed" else q.repeat(4 * S, 1), tokens=tokens.reshape(-1),
                 parents=torch.tensor([-1, 0, 0, 0], dtype=torch.int32).repeat(S),
                 start=torch.arange(0, 4 * S + 1, 4, dtype=torch.int32), u=torch.rand(4 * S, 2, generator=g),
                 news=[4] * S, V=V, mode=mode, n=4)
        n_path, path, token = run(x)
        first = np.where(n_path > 1, tokens.numpy()[np.arange(S), path[:, 1].clip(0)], token)
        count = np.bincount(first, minlength=V)
        want = p.double().numpy() / float(p.sum())
        assert (np.abs(count - S * want) <= 4.5 * np.sqrt(S * want * (1 - want))).all(), (mode, count, S * want)


@pytest.mark.gpu
def test_strided_rows_padding_and_bad_entries():
    x = make(6, 7, 501, 2, seed=12, mode="iid")
    want = run(x)
    N = x["p"].shape[0]
    wide = torch.full((N, 640), float("nan"), device="cuda")
    wide2 = torch.full((N, 517), float("nan"), device="cuda")
    wide[:, 3:504] = x["p"].cuda()
    wide2[:, :501] = x["q"].cuda()
    op = mls.TreeVerify(6, N, 501, max_path=7)
    got = op(wide[:, 3:504], x["tokens"].cuda(), x["parents"].cuda(), x["start"].cuda(), x["u"].cuda(), draft=wide2[:, :501])
    assert all((a.cpu().numpy() == b).all() for a, b in zip(got, want))
    assert mls.mls_get_status() == 0
    # offsets out of order or past the nodes, a parent after its child, node 0 below something, a path too long
    start = x["start"].clone()
    start[3] = N + 5
    bad = dict(x, start=start)
    n_path, path, token = run(bad)
    assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ
    assert (n_path[2:4] == 0).all() and (token[2:4] == -1).all() and (path[2:4] == -1).all()
    keep = [0, 1, 4, 5]
    assert (n_path[keep] == want[0][keep]).all() and (token[keep] == want[2][keep]).all()
    n_path, _, _ = run(x, max_path=3)
    assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ
    assert all(k == 0 for k, n in zip(n_path, x["news"]) if n > 3)
    assert all((k > 0) == (n > 0) for k, n in zip(n_path, x["news"]) if n <= 3)


@pytest.mark.gpu
def test_rows_without_mass_and_with_nan():
    x = make(4, 3, 100, 1, seed=2, mode="fixed", ragged=False)
    x["p"][:] = 0.0
    n_path, _, token = run(x)
    assert (n_path == 1).all() and (token == -1).all()
    x["p"][:] = float("nan")
    n_path, _, token = run(x)
    assert (n_path == 1).all() and (token == -1).all()


@pytest.mark.gpu
def test_the_same_answer_every_time_and_in_a_graph():
    x = make(3, 30, 40001, 3, seed=21, mode="distinct", ragged=False)
    args = [t.cuda() for t in (x["p"], x["tokens"], x["parents"], x["start"], x["u"])]
    q = x["q"].cuda()
    op = mls.TreeVerify(3, 90, 40001, max_path=30, replace=False)
    want = [t.clone() for t in op(*args, draft=q)]
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
        op(*args, draft=q)
    for _ in range(5):
        for t in (op.n_path, op.path, op.next_token):
            t.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((op.n_path, op.path, op.next_token), want))
    check(x, [t.cpu().numpy() for t in want])


def test_refusals():
    """What the host can see is refused before any launch (no GPU)."""
    import ctypes

    L = B.lib()
    p = ctypes.c_void_p(0x1000)

    def call(n=2, N=8, V=100, lt=100, ld=100, max_path=8, target=p, draft=p, tokens=p, out=p):
        pr = B.mls_tree_problem(n, N, V, lt, ld, 1, max_path)
        return L.mls_tree_verify(ctypes.byref(pr), target, draft, tokens, p, p, p, out, p, p, None)

    assert call(n=-1) == call(N=-1) == call(V=0) == call(V=1 << 31) == B.MLS_ERR_ARG
    assert call(max_path=0) == call(max_path=257) == B.MLS_ERR_ARG
    assert call(lt=99) == call(ld=99) == call(lt=1 << 40) == B.MLS_ERR_ARG
    assert call(target=None) == call(tokens=None) == call(out=None) == B.MLS_ERR_ARG
    assert call(target=ctypes.c_void_p(0x1002)) == B.MLS_ERR_ALIGN
    assert call(n=0, target=None) == B.MLS_OK
    assert L.mls_tree_verify(None, p, p, p, p, p, p, p, p, p, None) == B.MLS_ERR_ARG
    t = torch.zeros(8, 100)
    with pytest.raises(ValueError):
        B.mls_tree_verify(t, None, t, t, t, t, t, t[:, :4], t)  # not on the GPU
    with pytest.raises(ValueError):
        mls.TreeVerify(2, 8, 100, device="cpu")


def test_the_definition_itself():
    """By hand: V = 2, q = (0.8, 0.2), p = (0.5, 0.5): token 0 is accepted iff u < 0.625, and the residual
    after its refusal has all mass on token 1."""
    p, q = np.array([[0.5, 0.5], [0.3, 0.7]]), np.array([[0.8, 0.2], [0.5, 0.5]])
    for u, want in ((0.62, ([0, 1], 1)), (0.63, ([0], 1))):
        path, nxt, _ = walk(p, q, [0, 0], [-1, 0], np.array([[0.0, 0.01], [u, 0.4]]), "iid")
        assert (path, nxt) == want
