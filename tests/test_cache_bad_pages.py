"""A table that holds what is no page of the cache: compact and fork leave such an entry out, as it was to the
last bit, and raise the status; the entries beside it are served."""
import pytest
import torch

import paper_2608_09703_gb300 as mls
from test_cache import BAD, i32, pair, same


@pytest.fixture(autouse=True)
def clean_status(request):
    """Each test begins with no status of another."""
    if "gpu" in request.keywords:
        mls.mls_get_status()


# One block moves and closes an entry; several move it, and a second kernel closes it.
SIZES = [(1, 60, 8, 1, 8, 8, 9), (28, 40, 16, 2, 64, 8, 9)]
NO_PAGES = [-1, -7, 60, 1 << 30]


def filled(sizes, lens, more):
    """Sequences of lens tokens, with pages for `more` behind them, in the cache and in its model."""
    c, m = pair(*sizes, dtype=torch.bfloat16)
    ids = list(range(len(lens)))
    for m_call, c_call in ((m.reserve, c.reserve), (lambda i, n: m.compact(i, n, None), lambda n: c.compact(n))):
        m_call(ids, lens)
        c_call(i32(lens))
    m.reserve(ids, more)
    c.reserve(i32(more))
    same(c, m)
    return c, m


def spoil(c, m, row, col, page):
    m.rows[row][col] = page
    c.table[row, col] = page


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("page", NO_PAGES)
# columns 1 .. 4 of a row hold what is behind its len; the path reads columns 1 to 3 and writes 1 and 2
@pytest.mark.parametrize("col", [1, 2, 3, 4])
@pytest.mark.parametrize("with_path", [True, False])
def test_compact(sizes, page, col, with_path):
    ps = sizes[2]
    lens, more = [ps + 3, ps + 3, 2 * ps], [3 * ps] * 3
    c, m = filled(sizes, lens, more)
    spoil(c, m, 1, col, page)
    path = [sorted({0, 1, 3, ps - 4, ps - 2, ps, ps + 2, 2 * ps - 5, 3 * ps - 4})] * 3
    keep = [len(path[0])] * 3
    m.compact([0, 2], [keep[0], keep[2]], [path[0], path[2]] if with_path else None)
    m.status |= BAD
    c.compact(i32(keep), i32(path) if with_path else None)
    same(c, m)
    # the same with its page back in place
    spoil(c, m, 1, col, next(p for p in range(m.pages) if m.refs[p] and not any(p in r for r in m.rows)))
    m.compact([1], [keep[1]], path[1:2] if with_path else None)
    c.compact(i32(keep[1:2]), i32(path[1:2]) if with_path else None, i32([1]))
    same(c, m)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES)
def test_compact_of_a_path_of_several_turns(sizes):
    """More path tokens than a block looks at in one turn, the bad page only in the last of them."""
    layers, _, ps, heads, dim, seqs, _ = sizes
    most = 600 // ps + 2
    c, m = filled((layers, 2 * most + 4, ps, heads, dim, seqs, most), [3, 3], [590, 590])
    spoil(c, m, 0, len(m.rows[0]) - 1, -1)
    path = [list(range(1, 590)), list(range(1, 590))]
    m.compact([1], [589], path[1:])
    m.status |= BAD
    c.compact(i32([589, 589]), i32(path))
    same(c, m)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("page", NO_PAGES)
def test_fork(sizes, page):
    """Sources: a good one, one with a bad whole page, one whose partly filled page is bad, one of whole pages with
    a bad one, a good one."""
    ps = sizes[2]
    lens = [ps + 3, 2 * ps + 1, ps + 1, 2 * ps, 2]
    c, m = filled((sizes[0], sizes[1], ps, sizes[3], sizes[4], 10, 9), lens, [0] * 5)
    spoil(c, m, 1, 0, page)
    spoil(c, m, 2, 1, page)
    spoil(c, m, 3, 1, page)
    free = [p for p in range(m.pages) if m.refs[p] == 0]
    # Pages are handed out in the order of the entries; those of the entries left out are free again.
    m.fork([0], [5])
    m.refs[free[1]] = m.refs[free[2]] = 1
    m.fork([4], [9])
    m.refs[free[1]] = m.refs[free[2]] = 0
    m.status |= BAD
    assert m.rows[9] == [free[3]]
    c.fork(i32([0, 1, 2, 3, 4]), i32([5, 6, 7, 8, 9]))
    same(c, m)


@pytest.mark.gpu
@pytest.mark.parametrize("page", NO_PAGES)
def test_a_bad_page_in_front_of_len_or_given_back(page):
    """Compact neither reads nor writes the pages of what is kept already; free gives back the pages that are some."""
    c, m = filled(SIZES[0], [19, 5], [10, 3])
    good = m.rows[0][0]
    spoil(c, m, 0, 0, page)
    m.compact([0], [3], [[1, 2, 9]])
    c.compact(i32([3]), i32([[1, 2, 9]]))
    same(c, m)
    m.rows[0][0] = good
    m.free([0, 1])
    m.refs[good] = 1
    m.status |= BAD
    c.free()
    same(c, m)
