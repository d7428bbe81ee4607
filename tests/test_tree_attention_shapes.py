"""Tree attention where its tiles end: groups of heads that do not divide a tile, or are larger than one, entries
of a few rows and of many, single tokens over long caches split over the card.  Tolerances as in
test_tree_attention.py."""
import pytest
import torch

import paper_2608_09703_gb300 as mls
from test_tree_attention import BF16, F32, cache_of, check, make, run, run_and_check, visible

# lens, news, q_heads, kv_heads, dim, page
GROUPS = [
    ([40, 3], [3, 2], 130, 1, 64, 16), ([200], [3], 256, 1, 128, 32), ([9, 150], [2, 5], 192, 2, 72, 8),
    ([140], [5], 127, 1, 128, 16), ([64, 64], [4, 3], 96, 1, 40, 64), ([300], [20], 128, 1, 128, 128),
    ([33, 257], [9, 30], 18, 2, 128, 16), ([129], [50], 65, 1, 64, 8),
]


@pytest.mark.gpu
@pytest.mark.parametrize("tree", [True, False])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", GROUPS)
def test_groups_of_heads(shape, dtype, tree):
    run_and_check(make(*shape, dtype, seed=7, tree=tree))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("dim", [8, 24, 32, 56, 64, 72, 88, 96, 104, 120, 128])
def test_widths(dim, dtype):
    run_and_check(make([130, 0, 63], [7, 3, 20], 6, 2, dim, 16, dtype, seed=dim))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("group", [1, 4, 12])
def test_pages_and_groups_for_single_tokens(page, group, dtype):
    lens = [0, 1, 62, 63, 64, 65, 126, 127, 128, 129, 1000]
    run_and_check(make(lens, [1] * len(lens), 2 * group, 2, 64, page, dtype, seed=page + group, tree=False))


@pytest.mark.gpu
def test_a_width_of_four_in_fp32():
    run_and_check(make([70, 5], [6, 2], 4, 2, 4, 8, F32, seed=2))


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [2, 16])
def test_a_long_fp32_cache(heads):
    """Pieces of many CTAs joined, in items of 4 and of 16 rows."""
    run_and_check(make([60000, 100], [2, 1], heads, 1, 128, 64, F32))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_lengths_of_prompts(dtype):
    """Runs of items with as many tiles: chains whose items end on either side of a tile's end."""
    for news in ([129, 64, 63, 1, 300], [257, 128, 511]):
        lens = [(37 * i * i + 11) % 200 for i in range(len(news))]
        run_and_check(make(lens, news, 6, 2, 64, 16, dtype, seed=len(news), tree=False))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_empty_entries_around_others(dtype):
    run_and_check(make([5, 0, 300, 8, 0, 90], [0, 0, 4, 0, 0, 6], 4, 2, 64, 16, dtype, seed=5))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_same_answer_every_time(dtype):
    """No sum depends on which CTA comes first."""
    x = make([900, 20, 333, 4100], [9, 40, 3, 17], 8, 2, 128, 16, dtype, seed=11)
    c = cache_of(x)
    out, lse, _ = run(x, c=c)
    for _ in range(5):
        again, lse2, _ = run(x, c=c)
        assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_sequences_whose_nodes_all_take_no_part(dtype):
    x = make([100, 100, 30], [5, 140, 6], 4, 2, 64, 16, dtype, seed=12)
    x["parents"][5:145] = -2
    out, lse, scale = run(x)
    check(x, out, lse, scale)
    assert (out[5:145] == 0).all() and torch.isinf(lse[5:145]).all()
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,tree", [(1, False), (16, True), (70, True)])
def test_many_long_sequences(n, tree, dim):
    """Ranges of many tiles that end in others' midst, their last tiles masked: a warp that comes early to a tile with a
    mask must not touch what the ring holds before it."""
    g = torch.Generator().manual_seed(n + dim)
    lens = [3000] + [int(3000 * float(torch.rand(1, generator=g))) for _ in range(59)]
    run_and_check(make(lens, [n] * 60, 8, 2, dim, 32, BF16, seed=n, tree=tree))


@pytest.mark.gpu
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_heads", [8, 24])
def test_many_short_sequences(q_heads, dim):
    """Many short pieces of work a CTA, some with two row tiles: those that are taken side by side, and their neighbours."""
    g = torch.Generator().manual_seed(dim + q_heads)
    lens = [int(700 * float(torch.rand(1, generator=g)) ** 3) for _ in range(200)]
    news = [int(torch.randint(0, 8, (1,), generator=g)) for _ in range(200)]
    news[50], news[51], news[120] = 100, 200, 60
    run_and_check(make(lens, news, q_heads, 4, dim, 16, BF16, seed=dim, unused=0.1))


@pytest.mark.gpu
def test_infinite_values_in_many_short_sequences():
    """Each sequence's node 2 holds an infinite value: its column is infinite for the nodes that see it, nothing else is."""
    n, S = 9, 120
    g = torch.Generator().manual_seed(0)
    lens = [int(300 * float(torch.rand(1, generator=g))) for _ in range(S)]
    x = make(lens, [n] * S, 16, 8, 64, 16, BF16, seed=3, forest=0.0)
    for b in range(S):
        pos = lens[b] + 2
        x["v"][0, x["table"][b, pos // 16].long(), :, pos % 16, 3] = float("inf")
    for _ in range(5):
        out, lse, _ = run(x)
        assert mls.mls_get_status() == 0 and torch.isfinite(lse).all()
        for b in range(S):
            sees = visible(x, b)[:, lens[b] + 2]
            mine = out[b * n:(b + 1) * n]
            assert (mine[sees][..., 3] == float("inf")).all() and torch.isfinite(mine[~sees]).all(), b
            assert torch.isfinite(mine[..., [d for d in range(64) if d != 3]]).all(), b
