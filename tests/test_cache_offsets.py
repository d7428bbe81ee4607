"""Offsets of an append that go back or leave the tokens: the entries whose own break the rule are left out and raise
the status, whether a token would have come to them or not; the others get their tokens."""
import pytest
import torch

import paper_2608_09703_gb300 as mls
from test_cache import BAD, i32, pair, same


@pytest.fixture(autouse=True)
def clean_status(request):
    """Each test begins with no status of another."""
    if "gpu" in request.keywords:
        mls.mls_get_status()


# start, N, the entries that are left out
CASES = [
    ([0, 4, 2, 6], 6, [1, 2]),            # 1 goes back, 2 begins before the end of 0
    ([0, 4, 2, 6, 9], 9, [1, 2]),
    ([-3, 2, 5, 5], 5, [0]),
    ([0, 3, 7, 9], 8, [2]),               # past the tokens
    ([5, 2, 7, 8], 8, [0, 1]),
    ([0, 8, 2, 4, 6], 9, [1, 2, 3]),      # 3 does not go back by itself
    ([0, 0, 9, 9], 4, [1, 2]),            # an empty entry behind the last token
    ([2, 2, 2, 1], 5, [2]),               # no entry has a token
    ([0, 1 << 30, 3, 5], 5, [0, 1, 2]),
    ([-(1 << 31), (1 << 31) - 1, 0, 2], 3, [0, 1, 2]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("layer", [None, 1])
@pytest.mark.parametrize("listed", [True, False])
@pytest.mark.parametrize("start,N,out", CASES)
def test_offsets(start, N, out, listed, layer):
    n = len(start) - 1
    c, m = pair(2, 40, 8, 2, 16, 6, 4, dtype=torch.bfloat16)
    ids = [i + 1 if listed else i for i in range(n)]
    dev = i32(ids) if listed else None
    m.reserve(ids, [20] * n)
    c.reserve(i32([20] * n), dev)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(*((2, N) if layer is None else (N,)), 2, 16, generator=g).bfloat16() for _ in range(2))
    for e, i in enumerate(ids):
        if e not in out:
            one = range(start[e], start[e + 1])
            pick = (lambda x: x[:, one]) if layer is None else (lambda x: x[one])
            m.append([i], [0, len(one)], pick(k), pick(v), layer)
    m.status |= BAD
    c.append(k.cuda(), v.cuda(), i32(start), layer=layer, seqs=dev)
    same(c, m)


@pytest.mark.gpu
def test_many_entries():
    """More entries than a block has threads, most of them empty, and tokens behind the last."""
    n = 700
    c, m = pair(1, 900, 8, 1, 8, n, 2, dtype=torch.float32)
    g = torch.Generator().manual_seed(2)
    more = [int(torch.randint(0, 5, (1,), generator=g)) * (i % 3 == 0) for i in range(n)]
    start = [0]
    for x in more:
        start.append(start[-1] + x)
    N = start[-1] + 3
    k, v = (torch.randn(1, N, 1, 8, generator=g) for _ in range(2))
    m.reserve(list(range(n)), more)
    c.reserve(i32(more))
    m.append(list(range(n)), start, k, v, None)
    c.append(k.cuda(), v.cuda(), i32(start))
    same(c, m)
    # one offset in the middle a token too far: its entry takes a token of the next, which begins one later
    start[300] += 1
    start[301] = start[300] - 2  # and the next goes back
    left = {300} | {i for i in range(301, n) if start[i] < start[300]}
    for i in range(n):
        if i not in left and start[i + 1] > start[i]:
            one = range(start[i], start[i + 1])
            m.append([i], [0, len(one)], k[:, one], v[:, one], None)
    m.status |= BAD
    c.append(k.cuda(), v.cuda(), i32(start))
    same(c, m)
