"""The module's calls on a cache, tree attention and tree verification, beside the classes' methods that make the same
calls: the same state and outputs to the last bit, and the same refusals."""
import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from test_cache import i32

STATE = ("k", "v", "table", "len", "held", "refs", "free_bits")


def same(a, b):
    for name in STATE:
        x, y = getattr(a, name), getattr(b, name)
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), name
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cache(dtype):
    """`a` by the class, `b` by the module's calls."""
    a, b = (mls.PagedCache(2, 40, 16, 2, 64, 6, 5, dtype=dtype) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(1)
    for x, y in ((a.k, b.k), (a.v, b.v)):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        y.copy_(x)
    B.mls_cache_reset(b.c)
    same(a, b)
    for seqs in (None, i32([1, 3])):
        count, start = i32([30, 9]), i32([0, 20, 29])
        fused = torch.randn(2, 31, 7, 64, generator=g, device="cuda").to(dtype)
        k, v = fused[:, :, 1:3], fused[:, :, 5:7]
        a.reserve(count, seqs)
        B.mls_cache_reserve(b.c, seqs, count)
        same(a, b)
        a.append(k, v, start, seqs=seqs)
        B.mls_cache_append(b.c, -1, seqs, start, k, v)
        a.append(k[1].contiguous(), v[0].contiguous(), start, layer=1, seqs=seqs)
        B.mls_cache_append(b.c, 1, seqs, start, k[1].contiguous(), v[0].contiguous())
        same(a, b)
        keep, path = i32([4, 2]), i32([[0, 3, 7, 19], [1, 8, -1, -1]])
        a.compact(keep, path, seqs)
        B.mls_cache_compact(b.c, seqs, keep, path)
        same(a, b)
        a.reserve(i32([3, 3]), seqs)
        B.mls_cache_reserve(b.c, seqs, i32([3, 3]))
        a.compact(i32([3, 1]), None, seqs)
        B.mls_cache_compact(b.c, seqs, i32([3, 1]))
        same(a, b)
    src, dst = i32([1, 0]), i32([2, 5])
    a.fork(src, dst)
    B.mls_cache_fork(b.c, src, dst, b.ws)
    same(a, b)
    a.copy(i32([0, 1]), i32([30, 31]))
    B.mls_cache_copy(b.c, b.c, i32([0, 1]), i32([30, 31]))
    same(a, b)
    a.free(i32([1, 5]))
    B.mls_cache_free(b.c, 2, i32([1, 5]))
    same(a, b)
    a.free()
    B.mls_cache_free(b.c, 6, None)
    same(a, b)
    assert not b.refs.any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("listed", [True, False])
@pytest.mark.parametrize("tree", [True, False])
def test_tree_attention(dtype, listed, tree):
    g = torch.Generator(device="cuda").manual_seed(2)
    c = mls.PagedCache(2, 60, 16, 2, 64, 3, 20, dtype=dtype)
    c.k.copy_(torch.randn(c.k.shape, generator=g, device="cuda"))
    c.v.copy_(torch.randn(c.v.shape, generator=g, device="cuda"))
    c.reserve(i32([200, 17, 300]))
    c.compact(i32([200, 17, 300]))
    c.reserve(i32([9] * 3))
    seqs, start = i32([2, 0]) if listed else None, i32([0, 9, 14])
    q = torch.randn(14, 10, 64, generator=g, device="cuda").to(dtype)[:, 1:7]
    parents = i32([-1, 0, 0, 1, 3, -2, 2, 6, 6, -1, 0, 1, 2, 0]) if tree else None
    op = mls.TreeAttention(c, 2, 14, 6, 0.2)
    want = op(q, start, parents, 1, seqs)
    out, lse, ws = torch.zeros_like(op.out), torch.zeros_like(op.lse), torch.empty_like(op.ws)
    assert ws.numel() == B.mls_tree_attention_workspace_size(c.c, 2, 14, 6)
    B.mls_tree_attention(c.c, 1, seqs, start, parents, q, 0.2, out, lse, ws)
    assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and out.any()
    assert mls.mls_get_status() == 0
    for kw in (dict(out=out[:13]), dict(lse=lse.double()), dict(start=start.long()), dict(q=q[..., :32]),
               dict(q=q.transpose(0, 1)), dict(ws=ws.cpu()), dict(parents=i32([0]))):
        x = dict(start=start, q=q, out=out, lse=lse, ws=ws, parents=parents) | kw
        with pytest.raises((TypeError, ValueError)):
            B.mls_tree_attention(c.c, 1, seqs, x["start"], x["parents"], x["q"], 0.2, x["out"], x["lse"], x["ws"])


@pytest.mark.gpu
@pytest.mark.parametrize("drafted", [True, False])
@pytest.mark.parametrize("replace", [True, False])
def test_tree_verify(drafted, replace):
    g = torch.Generator(device="cuda").manual_seed(3)
    V, N = 501, 14
    wide = torch.rand(2, N, V + 11, generator=g, device="cuda")
    target, draft = (x / x.sum(1, keepdim=True) for x in wide[:, :, :V])
    wide[:, :, :V] = torch.stack((target, draft))
    target, draft = wide[0, :, :V], wide[1, :, :V]
    tokens = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    parents = i32([-1, 0, 0, 1, 3, -2, 2, 6, 6, -1, 0, 0, 0, 1])
    start, u = i32([0, 9, 14]), torch.rand(N, 2, generator=g, device="cuda")
    op = mls.TreeVerify(2, N, V, max_path=9, replace=replace)
    want = op(target, tokens, parents, start, u, draft=draft if drafted else None)
    got = i32([7, 7]), i32([[7] * 9] * 2), i32([7, 7])
    B.mls_tree_verify(target, draft if drafted else None, tokens, parents, start, u, *got, replace=replace)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert mls.mls_get_status() == 0


def test_refusals():
    """Tensors that are none of a GPU's never reach the library (no GPU)."""
    c, x = B.mls_cache(2, 10, 16, 2, 64, B.MLS_BF16, 4, 4), torch.zeros(2, dtype=torch.int32)
    rows = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: B.mls_cache_reserve(c, None, x), lambda: B.mls_cache_reserve(c, None, x.long()),
                 lambda: B.mls_cache_compact(c, None, x), lambda: B.mls_cache_fork(c, x, None, None),
                 lambda: B.mls_cache_free(c, 2, x), lambda: B.mls_cache_copy(c, c, x, x),
                 lambda: B.mls_cache_append(c, 0, None, x, rows, rows),
                 lambda: B.mls_tree_attention(c, 0, None, x, None, rows, 0.1, rows, rows, None)):
        with pytest.raises((TypeError, ValueError)):
            call()
