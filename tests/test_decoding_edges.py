"""Calls at the ends of the decoding operators' ranges: one large entry among empty ones, which an average over the entries
does not show, and the largest vocabulary."""
import pytest
import torch

import paper_2608_09703_gb300 as mls
from test_cache import i32
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
