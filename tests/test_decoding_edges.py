"""Calls at the ends of the decoding operators' ranges: one large entry among empty ones, which an average over the entries
does not show, the largest vocabulary, forks into the first sequences, a process whose first call is captured."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from test_cache import BAD, i32, pair, same
from test_tree_attention import BF16, F32, make, run_and_check


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("at", [0, 200, 255])
def test_one_tree_among_empty_entries(at, tree, dtype):
    """256 nodes of 4 heads a key/value head, 255 entries without nodes: 4 rows an entry on average."""
    lens, news = [30 * (b % 7) for b in range(256)], [0] * 256
    news[at] = 256
    run_and_check(make(lens, news, 8, 2, 64, 16, dtype, seed=at, tree=tree))


@pytest.mark.gpu
@pytest.mark.parametrize("drafted", [True, False])
def test_the_largest_vocabulary(drafted):
    """Two nodes over 2^31 - 1 tokens.  Node 0's child is token 7, where r is 0, so it is refused; then 3/4 of what is left
    lies at the last token, which a draw of 0.25 and more finds."""
    V = (1 << 31) - 1
    p = torch.zeros(2, V, device="cuda")
    p[0, 1 << 20], p[0, V - 1] = 0.25, 0.75
    q = None
    if drafted:
        q = torch.zeros(2, V, device="cuda")
        q[0, 7] = 1.0
    op = mls.TreeVerify(1, 2, V, max_path=2)
    for draw, token in ((0.2, 1 << 20), (0.25, V - 1), (0.9, V - 1)):
        u = torch.tensor([[0.5, draw], [0.5, 0.5]], device="cuda")
        n_path, path, nxt = op(p, i32([0, 7]), i32([-1, 0]), i32([0, 2]), u, draft=q)
        assert n_path.tolist() == [1] and path.tolist() == [[0, -1]] and nxt.tolist() == [token]
    # accepted, and drawn from the child's row
    p[0].zero_()
    p[0, V - 1] = p[1, V - 2] = 1.0
    if drafted:
        q[0, 7], q[0, V - 1] = 0.0, 1.0
    n_path, path, nxt = op(p, i32([0, V - 1]), i32([-1, 0]), i32([0, 2]), u, draft=q)
    assert n_path.tolist() == [2] and path.tolist() == [[0, 1]] and nxt.tolist() == [V - 2]
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
def test_fork_into_the_first_sequences():
    """No list of children: sequences 0, 1, ...; one of them is a source too, empty as all children have to be."""
    c, m = pair(2, 40, 16, 2, 64, 7, 5, dtype=torch.bfloat16)
    for ids, count in (([4, 5, 6], [33, 16, 7]),):
        m.reserve(ids, count)
        c.reserve(i32(count), i32(ids))
        m.compact(ids, count, None)
        c.compact(i32(count), None, i32(ids))
    m.fork([5, 4, 6, 1], [0, 1, 2, 3])
    B.mls_cache_fork(c.c, i32([5, 4, 6, 1]), None, c.ws)
    same(c, m)
    assert m.rows[3] == []
    # the first is not empty any more: left out, the fourth is served
    m.fork([4, 4, 4, 1], [0, 1, 2, 3])
    assert m.status == BAD
    B.mls_cache_fork(c.c, i32([4, 4, 4, 1]), None, c.ws)
    same(c, m)
    assert m.len[3] == 33


CAPTURE = r"""
import sys
sys.path.insert(0, {root!r})
import torch
import paper_2608_09703_gb300 as mls
g = torch.Generator(device="cuda").manual_seed(1)
p, q = (torch.softmax(torch.randn(12, 9001, generator=g, device="cuda"), 1) for _ in range(2))
tokens = torch.randint(0, 9001, (12,), generator=g, device="cuda", dtype=torch.int32)
parents = torch.tensor([-1, 0, 0, 1, 2, 2] * 2, dtype=torch.int32, device="cuda")
start = torch.tensor([0, 6, 12], dtype=torch.int32, device="cuda")
u = torch.rand(12, 2, generator=g, device="cuda")
op = mls.TreeVerify(2, 12, 9001, max_path=6)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    op(p, tokens, parents, start, u, draft=q)
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (op.n_path, op.path, op.next_token)]
want = op(p, tokens, parents, start, u, draft=q)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, want)) and mls.mls_get_status() == 0
print("CAPTURED")
"""


@pytest.mark.gpu
def test_first_call_of_a_process_inside_a_capture():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CAPTURE.format(root=root)], capture_output=True, text=True, timeout=240)
    assert r.returncode == 0 and "CAPTURED" in r.stdout, r.stdout + r.stderr
