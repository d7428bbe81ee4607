"""Attention of a tree's nodes over a paged cache against the definition in 64 bits, row by row.

Tolerances.  bf16: the output is rounded once, by 2^-8 of itself at most, and each weight exp(z - m) once before
it meets its value, by 2^-8 of it: |error| <= 2^-8 |out| + 2^-8 sum_j w_j |v_j| plus what fp32 sums add.  fp32
sums: products of head_dim terms (|z| off by dim 2^-24 sum |q_i k_i| scale, and by 2^-22 |z| log2(e) of the
exponent's argument), exponentials by 2^-22, sums over n weights by at most n 2^-24 each: together the weights
move by E = 2^-22 + n 2^-24 + 2 max(dz) relative, and so does sum_j w_j |v_j|.  lse moves by max(dz) + n 2^-24."""
import ctypes
import math

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B

BF16, F32 = torch.bfloat16, torch.float32


def make(lens, news, q_heads, kv_heads, dim, page, dtype, seed=0, tree=True, spread=3, unused=0.0, layers=1, layer=0,
         q_scale=2.0, garbage=float("nan"), forest=0.1):
    """A cache whose pages lie anywhere, all that no sequence holds full of `garbage`, and nodes' queries."""
    g = torch.Generator().manual_seed(seed)
    S, N = len(lens), sum(news)
    held = [-(-(a + b) // page) for a, b in zip(lens, news)]
    pages, most = sum(held) + 3, max(held + [1])
    order = torch.randperm(pages, generator=g).int()
    k = torch.full((layers, pages, kv_heads, page, dim), garbage).to(dtype)
    v = k.clone()
    table = torch.full((S, most), -1, dtype=torch.int32)
    keys, values, at = [], [], 0
    for b in range(S):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
        total = lens[b] + news[b]
        kb, vb = (torch.randn(total, kv_heads, dim, generator=g).to(dtype) for _ in range(2))
        for t in range(0, total, page):
            m = min(page, total - t)
            k[layer, table[b, t // page].long(), :, :m] = kb[t:t + m].transpose(0, 1)
            v[layer, table[b, t // page].long(), :, :m] = vb[t:t + m].transpose(0, 1)
        keys.append(kb)
        values.append(vb)
    q = (torch.randn(N, q_heads, dim, generator=g) * q_scale).to(dtype)
    parents = None
    if tree:
        parents = torch.empty(N, dtype=torch.int32)
        i = 0
        for n in news:
            for j in range(n):
                up = j - 1 - int(torch.randint(0, max(1, min(j, spread)), (1,), generator=g))
                r = float(torch.rand(1, generator=g))
                parents[i] = -2 if r < unused else -1 if r < unused + forest else up
                i += 1
    start = [0]
    for n in news:
        start.append(start[-1] + n)
    return dict(lens=lens, news=news, q=q, k=k, v=v, table=table, keys=keys, values=values, parents=parents,
                start=torch.tensor(start, dtype=torch.int32), layer=layer, dtype=dtype, page=page,
                shape=(layers, pages, page, kv_heads, dim, S, most))


def visible(x, b):
    """[n, len + n] truth values."""
    have, n, at = x["lens"][b], x["news"][b], int(x["start"][b])
    see = torch.zeros(n, have + n, dtype=torch.bool)
    for i in range(n):
        if x["parents"] is None:
            see[i, :have + i + 1] = True
            continue
        up = x["parents"][at:at + n].tolist()
        if up[i] < -1:
            continue
        see[i, :have] = True
        j = i
        while j >= 0 and up[j] >= -1:
            see[i, have + j] = True
            j = up[j]
    return see


def check(x, out, lse, scale):
    dim, G = x["q"].shape[2], x["q"].shape[1] // x["k"].shape[2]
    half = torch.finfo(x["dtype"]).eps / 2 if x["dtype"] == BF16 else 0.0
    for b, n in enumerate(x["news"]):
        if n == 0:
            continue
        at, see = int(x["start"][b]), visible(x, b)
        K, V = x["keys"][b].double().repeat_interleave(G, 1), x["values"][b].double().repeat_interleave(G, 1)
        q = x["q"][at:at + n].double()
        total = K.shape[0]
        alive = see.any(1)
        K = torch.where(see.any(0)[:, None, None], K, 0.0)
        V = torch.where(see.any(0)[:, None, None], V, 0.0)
        z = torch.einsum("nhd,thd->hnt", q, K) * scale
        dz = torch.einsum("nhd,thd->hnt", q.abs(), K.abs()) * (abs(scale) * dim * 2.0 ** -24) + z.abs() * 2.0 ** -21
        hide = ~see[None]
        z = z.masked_fill(hide, -math.inf)
        want_lse = torch.logsumexp(z, 2)
        w = torch.exp(z - want_lse.masked_fill(~alive[None], 0.0)[..., None])
        worst = dz.masked_fill(hide, 0.0).amax(2)
        want = torch.einsum("hnt,thd->nhd", w, V)
        size = torch.einsum("hnt,thd->nhd", w, V.abs())
        move = (2.0 ** -22 + total * 2.0 ** -24 + 2 * worst).T[..., None]
        bound = half * want.abs() + (half + move) * size * (1 + half) + 1e-30
        got, gl = out[at:at + n].double(), lse[at:at + n].double()
        assert torch.equal(got[~alive], torch.zeros_like(got[~alive])) and (gl[~alive] == -math.inf).all()
        err = (got - want).abs()[alive]
        assert (err <= bound[alive]).all(), (b, float((err / bound[alive]).max()))
        lerr = (gl - want_lse.T).abs()[alive]
        lb = (worst.T + total * 2.0 ** -24 + 2.0 ** -22 * (1 + want_lse.T.abs()))[alive]
        assert (lerr <= lb).all(), (b, float((lerr / lb).max()))


def cache_of(x):
    layers, pages, page, kv, dim, S, most = x["shape"]
    c = mls.PagedCache(layers, pages, page, kv, dim, S, most, dtype=x["dtype"])
    c.k.copy_(x["k"])
    c.v.copy_(x["v"])
    c.table.copy_(x["table"])
    c.len.copy_(torch.tensor(x["lens"], dtype=torch.int32))
    c.held.copy_((x["table"] >= 0).sum(1))
    return c


def run(x, scale=None, c=None, **kw):
    c = c or cache_of(x)
    op = mls.TreeAttention(c, len(x["news"]), x["q"].shape[0], x["q"].shape[1], scale)
    out, lse = op(x["q"].cuda(), x["start"].cuda(), None if x["parents"] is None else x["parents"].cuda(), x["layer"], **kw)
    torch.cuda.synchronize()
    return out.cpu(), lse.cpu(), op.scale


def run_and_check(x, status=0, **kw):
    out, lse, scale = run(x, **kw)
    assert mls.mls_get_status() == status
    check(x, out, lse, scale)
    return out, lse


# lens, news, q_heads, kv_heads, dim, page
SHAPES = [
    ([0], [1], 1, 1, 64, 8), ([1], [1], 4, 1, 128, 16), ([0, 5, 127, 128, 129], [1, 1, 1, 1, 1], 8, 2, 128, 16),
    ([700], [8], 16, 4, 64, 16), ([300, 0, 1111], [16, 3, 16], 32, 8, 128, 16), ([255, 64], [64, 33], 32, 8, 128, 64),
    ([130], [256], 4, 2, 128, 32), ([1000, 17, 383], [9, 40, 100], 6, 2, 72, 8), ([500], [70], 21, 3, 96, 128),
    ([513, 250], [5, 0], 14, 2, 40, 256), ([77, 0, 0, 900], [2, 0, 7, 1], 5, 5, 8, 16), ([2000], [3], 16, 1, 104, 64),
    ([120, 121, 122, 123, 124, 125, 126, 127], [8, 7, 6, 5, 4, 3, 2, 1], 10, 2, 128, 8), ([5000], [31], 64, 8, 128, 32),
]


@pytest.mark.gpu
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_definition(shape, dtype, tree):
    run_and_check(make(*shape, dtype, seed=len(shape[0]) + shape[4], tree=tree))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lens,news", [([300, 20], [700, 130]), ([0], [1025]), ([129], [384])])
def test_prompts(lens, news, dtype):
    """Chains of more nodes than a tree may have: a prompt read behind what the cache holds."""
    run_and_check(make(lens, news, 8, 2, 128 if dtype == BF16 else 64, 16, dtype, tree=False))


@pytest.mark.gpu
def test_many_sequences():
    """More sequences and heads than there are SMs, lengths from none to some thousand."""
    g = torch.Generator().manual_seed(8)
    lens = [int(3000 * float(torch.rand(1, generator=g)) ** 3) for _ in range(70)]
    news = [int(torch.randint(0, 12, (1,), generator=g)) for _ in range(70)]
    run_and_check(make(lens, news, 8, 4, 64, 16, BF16))


@pytest.mark.gpu
def test_a_long_cache():
    run_and_check(make([70000, 33], [4, 2], 4, 1, 128, 64, BF16))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_what_a_node_does_not_see_may_hold_anything(dtype, what):
    """Keys and values of unused nodes, and of nodes on other branches."""
    x = make([200, 31], [40, 9], 8, 2, 128, 16, dtype, seed=3, unused=0.25, garbage=what)
    at = 0
    for b, n in enumerate(x["news"]):
        for i in range(n):
            if int(x["parents"][at + i]) == -2:
                pos = x["lens"][b] + i
                page, slot = x["table"][b, pos // 16].long(), pos % 16
                x["k"][0, page, :, slot] = what
                x["v"][0, page, :, slot] = what
        at += n
    run_and_check(x)
    # a branch whose values overflowed: its own nodes say so, the others are as they would be without it
    y = make([200], [30], 8, 2, 128, 16, dtype, seed=4, forest=0.0)
    want, wlse, _ = run(y)
    see = visible(y, 0)
    bad = 7
    pos = 200 + bad
    page, slot = y["table"][0, pos // 16].long(), pos % 16
    y["v"][0, page, :, slot, 3::5] = what
    y["v"][0, page, 1, slot, 0] = what
    out, lse, _ = run(y)
    blind = ~see[:, pos]
    assert blind.any() and see[:, pos].any()
    assert torch.equal(out[blind], want[blind]) and torch.equal(lse, wlse)
    hit = out[see[:, pos]][:, :, 3::5]
    assert (torch.isnan(hit) if math.isnan(what) else hit == what).all()
    clean = [d for d in range(1, 128) if d % 5 != 3]
    assert torch.isfinite(out[see[:, pos]][:, :, clean]).all()
    half = torch.finfo(dtype).eps
    assert ((out[see[:, pos]][:, :, clean].double() - want[see[:, pos]][:, :, clean].double()).abs()
            <= half * want[see[:, pos]][:, :, clean].double().abs() + 1e-30).all()
    y["k"][0, page, :, slot] = what
    out, lse, _ = run(y)
    assert torch.equal(out[blind], want[blind]) and torch.equal(lse[blind], wlse[blind])


@pytest.mark.gpu
def test_a_prompts_later_tokens_are_not_seen():
    y = make([100], [300], 4, 2, 128, 16, BF16, tree=False)
    want, wlse, _ = run(y)
    for pos in (100 + 150, 100 + 299):
        page, slot = y["table"][0, pos // 16].long(), pos % 16
        y["k"][0, page, :, slot] = float("nan")
        y["v"][0, page, :, slot] = float("inf")
    out, lse, _ = run(y)
    assert torch.equal(out[:150], want[:150]) and torch.equal(lse[:150], wlse[:150])
    assert torch.isnan(out[150:]).all() and torch.isnan(lse[150:]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_extreme_scores(dtype):
    """Scores of some hundred either way, a scale of 0 and a negative one."""
    x = make([400], [12], 8, 2, 64, 16, dtype, q_scale=60.0)
    run_and_check(x)
    run_and_check(x, scale=0.0)
    run_and_check(x, scale=-0.01)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layers_order_of_sequences_strides_and_padding(dtype):
    x = make([90, 300, 7, 64], [5, 9, 1, 17], 6, 2, 64, 16, dtype, layers=3, layer=2, seed=6)
    want, wlse = run_and_check(x)
    c = cache_of(x)
    # entries 3, 1, 1, 0 with the queries of a fused projection, tokens behind the last entry left alone
    order = [3, 1, 1, 0]
    rows = [torch.arange(int(x["start"][b]), int(x["start"][b + 1])) for b in order]
    pick = torch.cat(rows)
    N = len(pick) + 4
    fused = torch.full((N, 12, 64), float("nan"), dtype=dtype, device="cuda")
    fused[:len(pick), 2:8] = x["q"][pick].cuda()
    start = torch.tensor([0] + [len(r) for r in rows]).cumsum(0).int().cuda()
    parents = torch.cat([x["parents"][pick], torch.full((4,), 99)]).int().cuda()
    op = mls.TreeAttention(c, 4, N, 6)
    op.out.fill_(7.0)
    op.lse.fill_(7.0)
    out, lse = op(fused[:, 2:8], start, parents, 2, seqs=torch.tensor(order, dtype=torch.int32, device="cuda"))
    assert (out[len(pick):] == 7).all() and (lse[len(pick):] == 7).all()
    # how the keys are split over the card depends on the call, so sums may be ordered otherwise
    y = dict(x, q=x["q"][pick], lens=[x["lens"][b] for b in order], news=[x["news"][b] for b in order],
             keys=[x["keys"][b] for b in order], values=[x["values"][b] for b in order], parents=x["parents"][pick],
             start=start.cpu())
    check(y, out[:len(pick)].cpu(), lse[:len(pick)].cpu(), op.scale)
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_entries_that_do_not_fit(dtype):
    """A sequence that is none, offsets out of order, parents after their child, a table too short, a page that
    is none: raised, the nodes concerned without part, the others right."""
    x = make([50, 60, 70], [4, 5, 6], 4, 2, 64, 16, dtype, seed=9, forest=0.0)
    c = cache_of(x)
    out, lse, scale = run(x, c=c, seqs=torch.tensor([0, 3, 2], dtype=torch.int32, device="cuda"))
    assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ
    dead = slice(4, 9)
    assert (out[dead] == 0).all() and (lse[dead] == -math.inf).all()
    y = dict(x, parents=x["parents"].clone())
    y["parents"][dead] = -2
    check(y, out, lse, scale)
    # parents that are no parents count as -2
    z = dict(x, parents=x["parents"].clone())
    z["parents"][6], z["parents"][12], z["parents"][13] = 2, -5, 100
    out, lse, scale = run(z, c=c)
    assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ
    z["parents"][6] = z["parents"][12] = z["parents"][13] = -2
    check(z, out, lse, scale)
    # more tokens than the table has room for
    c.len[1] = c.table.shape[1] * 16 - 4
    out, lse, scale = run(x, c=c)
    assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ
    assert (out[dead] == 0).all()
    check(y, out, lse, scale)
    c.len[1] = -1
    out, lse, scale = run(x, c=c)
    assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ
    check(y, out, lse, scale)
    # a page that is none: keys and values of zeros
    c = cache_of(x)
    for wrong in (-1, c.table.max().item() + 1000, c.refs.numel()):
        c.table[2, 1] = wrong
        out, lse, scale = run(x, c=c)
        assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ
        w = dict(x, keys=list(x["keys"]), values=list(x["values"]))
        for name in ("keys", "values"):
            w[name][2] = w[name][2].clone()
            w[name][2][16:32] = 0
        check(w, out, lse, scale)
    # a tree of more nodes than one may have
    big = make([10, 12], [257, 3], 2, 1, 64, 16, dtype)
    out, lse, scale = run(big)
    assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ
    assert (out[:257] == 0).all() and (lse[:257] == -math.inf).all()
    big["parents"][:257] = -2
    check(big, out, lse, scale)


@pytest.mark.gpu
def test_two_streams_a_graph_and_changing_lengths():
    """Two objects on two streams; a captured call follows what the cache holds when it is replayed."""
    xs = [make([300, 20], [5, 9], 8, 2, 128, 16, BF16, seed=s) for s in (1, 2)]
    want = [run(x) for x in xs]
    ops = []
    for x in xs:
        c = cache_of(x)
        ops.append((mls.TreeAttention(c, 2, 14, 8), x["q"].cuda(), x["start"].cuda(), x["parents"].cuda(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for op, q, start, parents, s in ops:
            with torch.cuda.stream(s):
                op(q, start, parents)
    torch.cuda.synchronize()
    for (op, *_), (out, lse, _) in zip(ops, want):
        assert torch.equal(op.out.cpu(), out) and torch.equal(op.lse.cpu(), lse)
    op, q, start, parents, s = ops[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
        op(q, start, parents)
    for cut in (0, 17, 130):
        y = dict(xs[0], lens=[300 - cut, 20])
        y["keys"] = [xs[0]["keys"][0][:305 - cut], xs[0]["keys"][1]]
        y["values"] = [xs[0]["values"][0][:305 - cut], xs[0]["values"][1]]
        op.cache.len[0] = 300 - cut
        op.out.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(y, op.out.cpu(), op.lse.cpu(), op.scale)
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A cache of more than 2^32 values, its sequence's pages at the end of it."""
    pages, page, kv, dim = 4300, 256, 8, 128
    c = mls.PagedCache(4, pages, page, kv, dim, 1, 4)
    assert c.k.numel() > 1 << 32
    x = make([600], [9], 16, kv, dim, page, BF16, seed=5)
    c.table[0, :3] = torch.tensor([pages - 1, pages - 2, pages - 3], dtype=torch.int32, device="cuda")
    for i in range(3):
        src = x["table"][0, i].long()
        c.k[3, pages - 1 - i] = x["k"][0, src].cuda()
        c.v[3, pages - 1 - i] = x["v"][0, src].cuda()
    c.len[0] = 600
    out, lse, scale = run(dict(x, layer=3), c=c)
    check(x, out, lse, scale)
    assert mls.mls_get_status() == 0


def test_refusals():
    """What the host can see is refused before any launch (no GPU)."""
    L, P = B.lib(), 0x1000
    p = ctypes.c_void_p(P)

    def call(layer=0, n=2, N=8, heads=4, q=p, ld=256, scale=0.1, out=p, ws=p, size=1 << 40, seqs=p, dim=64,
             dtype=B.MLS_BF16, layers=2, pages=10, kv=2):
        c = B.mls_cache(layers, pages, 16, kv, dim, dtype, 4, 4, P, P, P, P, P, P, P)
        return L.mls_tree_attention(ctypes.byref(c), layer, n, seqs, p, p, N, heads, q, ld, scale, out, p, ws, size, None)

    for kw in (dict(layer=-1), dict(layer=2), dict(n=-1), dict(n=5, seqs=None), dict(N=-1), dict(heads=0), dict(heads=3),
               dict(q=None), dict(out=None), dict(ld=255), dict(ld=1 << 50), dict(scale=float("nan")),
               dict(scale=float("inf"))):
        assert call(**kw) == B.MLS_ERR_ARG, kw
    assert call(ld=260) == call(q=ctypes.c_void_p(P + 8)) == call(out=ctypes.c_void_p(P + 2)) == B.MLS_ERR_ALIGN
    assert call(dim=136, ld=1000) == call(layers=1 << 10, pages=1 << 20, kv=2) == B.MLS_ERR_UNSUPPORTED
    assert call(ws=None) == call(size=100) == B.MLS_ERR_WORKSPACE
    assert call(n=0, q=None) == call(N=0, q=None) == B.MLS_OK


def test_the_definition_itself():
    """By hand: one key of weight 1; two equal keys; a root beside another; an unused node."""
    x = make([1], [3], 1, 1, 8, 8, F32)
    x["parents"] = torch.tensor([-1, -1, 0], dtype=torch.int32)
    assert visible(x, 0).tolist() == [[True, True, False, False], [True, False, True, False], [True, True, False, True]]
    x["parents"] = torch.tensor([-1, -2, 1], dtype=torch.int32)
    assert visible(x, 0).tolist() == [[True, True, False, False], [False] * 4, [True, False, False, True]]
