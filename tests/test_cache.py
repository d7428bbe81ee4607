"""The paged cache against a model of it in plain Python: after every call the whole state has to be equal,
the pool's bits, the table, lengths, counts and the map of free pages."""
import ctypes
import random

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B

BAD, NONE = B.MLS_STATUS_BAD_SEQ, B.MLS_STATUS_NO_PAGES


class Model:
    def __init__(self, layers, pages, page_size, heads, dim, seqs, max_pages, dtype):
        self.ps, self.pages, self.seqs, self.most = page_size, pages, seqs, max_pages
        self.k = torch.zeros(layers, pages, heads, page_size, dim, dtype=dtype)
        self.v = torch.zeros_like(self.k)
        self.rows, self.len, self.refs, self.status = [[] for _ in range(seqs)], [0] * seqs, [0] * pages, 0

    def good(self, ids):
        """Which entries are strictly greater than all before them, and sequences of the cache."""
        top, out = -1, []
        for i in ids:
            ok = 0 <= i < self.seqs and i > top
            out.append(ok)
            if not ok:
                self.status |= BAD
            top = max(top, i)
        return out

    def take(self, wants):
        """Lowest free pages for each want, in order; those that cannot be met get None, and all after them."""
        free = [p for p in range(self.pages) if self.refs[p] == 0]
        out, at, short = [], 0, False
        for w in wants:
            short = short or at + w > len(free)
            if short:
                if w:
                    self.status |= NONE
                out.append(None if w else [])
                continue
            out.append(free[at:at + w])
            at += w
            for p in out[-1]:
                self.refs[p] = 1
        return out

    def reserve(self, ids, count):
        wants = []
        for i, ok, c in zip(ids, self.good(ids), count):
            need = 0
            if ok and c < 0:
                self.status |= BAD
            elif ok:
                pages = -(-(self.len[i] + c) // self.ps)
                if pages > self.most:
                    self.status |= NONE
                else:
                    need = max(0, pages - len(self.rows[i]))
            wants.append(need)
        for i, got in zip(ids, self.take(wants)):
            if got:
                self.rows[i] += got

    def append(self, ids, start, k, v, layer):
        status = self.status
        good = self.good(ids)
        self.status = status  # an entry is looked at for each of its tokens
        for e, i in enumerate(ids):
            if not good[e] and start[e + 1] > start[e]:
                self.status |= BAD
            for t in range(start[e], start[e + 1]):
                if not good[e]:
                    continue
                at = self.len[i] + t - start[e]
                if at // self.ps >= len(self.rows[i]):
                    self.status |= NONE
                    continue
                page, slot = self.rows[i][at // self.ps], at % self.ps
                for pool, new in ((self.k, k), (self.v, v)):
                    if layer is None:
                        pool[:, page, :, slot] = new[:, t]
                    else:
                        pool[layer, page, :, slot] = new[t]

    def compact(self, ids, keep, path):
        for e, (i, ok) in enumerate(zip(ids, self.good(ids))):
            if not ok:
                continue
            room = len(self.rows[i]) * self.ps - self.len[i]
            p = list(range(keep[e])) if path is None else list(path[e][:max(keep[e], 0)])
            if keep[e] < 0 or keep[e] > room or (path is not None and keep[e] > len(path[e])) or any(
                    a < 0 or a >= room for a in p) or any(a >= b for a, b in zip(p, p[1:])):
                self.status |= BAD
                continue
            for j, a in enumerate(p):
                src, dst = self.len[i] + a, self.len[i] + j
                for pool in (self.k, self.v):
                    pool[:, self.rows[i][dst // self.ps], :, dst % self.ps] = \
                        pool[:, self.rows[i][src // self.ps], :, src % self.ps].clone()
            self.len[i] += keep[e]
            self.drop(i, -(-self.len[i] // self.ps))

    def drop(self, i, to):
        for p in self.rows[i][to:]:
            self.refs[p] -= 1
        self.rows[i] = self.rows[i][:to]

    def fork(self, src, dst):
        plan, wants, empty = [], [], [not r for r in self.rows]
        for s, d, ok in zip(src, dst, self.good(dst)):
            fine = ok and 0 <= s < self.seqs and empty[d]
            if ok and not fine:
                self.status |= BAD
            plan.append((s, d, self.len[s]) if fine else None)
            wants.append(int(fine and self.len[s] % self.ps > 0))
        old = [list(r) for r in self.rows]
        for p, w, got in zip(plan, wants, self.take(wants)):
            if p is None or got is None:
                continue
            s, d, n = p
            self.rows[d] = old[s][:n // self.ps] + got
            self.len[d] = n
            for page in old[s][:n // self.ps]:
                self.refs[page] += 1
            if w:
                for pool in (self.k, self.v):
                    pool[:, got[0], :, :n % self.ps] = pool[:, old[s][n // self.ps], :, :n % self.ps]

    def free(self, ids):
        for i, ok in zip(ids, self.good(ids)):
            if ok:
                self.drop(i, 0)
                self.len[i] = 0


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same(c, m):
    assert torch.equal(c.k.cpu().view(torch.uint8), m.k.view(torch.uint8))
    assert torch.equal(c.v.cpu().view(torch.uint8), m.v.view(torch.uint8))
    assert c.len.tolist() == m.len and c.held.tolist() == [len(r) for r in m.rows]
    assert c.table.tolist() == [r + [-1] * (m.most - len(r)) for r in m.rows]
    assert c.refs.tolist() == m.refs
    bits = [b & 0xffffffff for b in c.free_bits.tolist()]
    assert [bits[p // 32] >> (p % 32) & 1 for p in range(m.pages)] == [int(r == 0) for r in m.refs]
    status, m.status = m.status, 0
    assert mls.mls_get_status() == status


def pair(*sizes, dtype):
    c, m = mls.PagedCache(*sizes, dtype=dtype), Model(*sizes, dtype)
    g = torch.Generator().manual_seed(1)
    for a, b in ((c.k, m.k), (c.v, m.v)):
        b.copy_(torch.randn(b.shape, generator=g))
        a.copy_(b)
    return c, m


# layers, pages, page_size, heads, dim, seqs, max_pages
SIZES = [((1, 33, 8, 1, 8, 5, 9), torch.bfloat16), ((3, 70, 16, 3, 72, 9, 12), torch.bfloat16),
         ((2, 40, 64, 2, 4, 6, 5), torch.float32), ((28, 20, 256, 2, 128, 4, 6), torch.bfloat16),
         ((2, 1500, 8, 5, 20, 40, 300), torch.float32), ((1, 1, 8, 1, 8, 1, 1), torch.bfloat16)]


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(len(SIZES)))
def test_random_calls(which):
    sizes, dtype = SIZES[which]
    layers, pages, ps, heads, dim, seqs, most = sizes
    c, m = pair(*sizes, dtype=dtype)
    same(c, m)
    rng, g = random.Random(which), torch.Generator().manual_seed(which)

    def entries(least=1):
        ids = sorted(rng.sample(range(seqs), rng.randint(min(least, seqs), seqs)))
        if rng.random() < 0.15:  # one that breaks the rule: out of order, twice, or none of the cache's
            at = rng.randrange(len(ids))
            ids.insert(at, rng.choice([ids[at], -1, seqs, ids[0]]))
            ids = ids[:seqs]
        return ids, None if ids == list(range(len(ids))) and rng.random() < 0.5 else i32(ids)

    for step in range(60):
        ids, dev = entries()
        what = rng.choice(["grow", "grow", "grow", "compact", "fork", "free"])
        if what == "grow":
            count = [rng.choice([0, 1, rng.randint(0, 3 * ps), rng.randint(0, ps)]) for _ in ids]
            if rng.random() < 0.1:
                count[0] = -1
            m.reserve(ids, count)
            c.reserve(i32(count), dev)
            same(c, m)
            more = [rng.randint(0, max(x, 0) + (rng.random() < 0.1)) for x in count]
            start = [0]
            for x in more:
                start.append(start[-1] + x)
            N = start[-1] + 2  # two tokens behind the last entry
            layer = rng.choice([None, rng.randrange(layers)])
            shape = (N, heads, dim) if layer is not None else (layers, N, heads, dim)
            k, v = (torch.randn(shape, generator=g).to(dtype) for _ in range(2))
            m.append(ids, start, k, v, layer)
            c.append(k.cuda(), v.cuda(), i32(start), layer=layer, seqs=dev)
        elif what == "compact":
            rooms = [len(m.rows[i]) * ps - m.len[i] if 0 <= i < seqs else 1 for i in ids]
            if rng.random() < 0.5:
                keep, path, dpath = [rng.randint(0, r) for r in rooms], None, None
            else:
                path = [sorted(rng.sample(range(r), rng.randint(0, min(r, 300)))) for r in rooms]
                keep = [len(p) for p in path]
                width = max(1, max(keep))
                path = [p + [-1] * (width - len(p)) for p in path]
                if rng.random() < 0.2 and keep[0] > 1:
                    path[0][1] = path[0][0]
                dpath = i32(path)
            if rng.random() < 0.1:
                keep[-1] = rng.choice([-1, rooms[-1] + 1, 1 << 30])
            m.compact(ids, keep, path)
            c.compact(i32(keep), dpath, dev)
        elif what == "fork":
            if dev is None:
                dev = i32(ids)
            src = [rng.choice([rng.randrange(seqs), rng.randrange(seqs), -1, seqs][:2 if rng.random() < 0.9 else 4]) for _ in ids]
            if rng.random() < 0.7:
                some = sorted({i for i in ids if 0 <= i < seqs and i not in src})[:2]
                m.free(some)
                if some:
                    c.free(i32(some))
            m.fork(src, ids)
            c.fork(i32(src), dev)
        else:
            m.free(ids)
            c.free(dev if dev is not None else i32(ids))
        same(c, m)
    m.free(list(range(seqs)))
    c.free()
    same(c, m)
    assert m.refs == [0] * pages


@pytest.mark.gpu
def test_many_entries_and_too_few_pages():
    """Over a thousand entries (several turns of the one block), and more wanted than there is."""
    c, m = pair(1, 3000, 8, 1, 8, 2500, 4, dtype=torch.bfloat16)
    rng = random.Random(4)
    ids = sorted(rng.sample(range(2500), 2100))
    ids[700], ids[1500] = ids[699], 5
    count = [rng.randint(0, 12) for _ in ids]
    m.reserve(ids, count)
    c.reserve(i32(count), i32(ids))
    same(c, m)
    keep = [min(x, 8 * len(m.rows[i])) for i, x in zip(ids, count)]
    m.compact(ids, keep, None)
    c.compact(i32(keep), None, i32(ids))
    same(c, m)
    m.reserve(list(range(2500)), [20] * 2500)
    c.reserve(i32([20] * 2500))
    same(c, m)
    src = [ids[rng.randrange(100)] for _ in range(2500)]
    m.fork(src, list(range(2500)))
    c.fork(i32(src), i32(list(range(2500))))
    same(c, m)
    m.free(list(range(1, 2500, 2)))
    c.free(i32(list(range(1, 2500, 2))))
    same(c, m)


@pytest.mark.gpu
def test_one_prompt_forked_many_times_with_too_few_pages():
    """The forks past the last free page are left out, the others not."""
    c, m = pair(2, 30, 16, 2, 64, 64, 8, dtype=torch.bfloat16)
    m.reserve([0], [77])
    c.reserve(i32([77]))
    m.compact([0], [77], None)
    c.compact(i32([77]))
    m.fork([0] * 63, list(range(1, 64)))
    c.fork(i32([0] * 63), i32(list(range(1, 64))))
    same(c, m)
    assert m.refs[0] == 26 and m.len.count(77) == 26
    m.free([0])
    c.free(i32([0]))
    same(c, m)
    # a whole number of pages needs no page of its own
    c, m = pair(2, 6, 16, 2, 64, 64, 8, dtype=torch.bfloat16)
    m.reserve([0], [96])
    c.reserve(i32([96]))
    m.compact([0], [96], None)
    c.compact(i32([96]))
    m.fork([0] * 63, list(range(1, 64)))
    c.fork(i32([0] * 63), i32(list(range(1, 64))))
    same(c, m)
    assert m.refs == [64] * 6


@pytest.mark.gpu
def test_strided_new_tokens_and_other_stream():
    """Keys and values as views of one fused projection; calls on a stream of their own."""
    c, m = pair(2, 20, 16, 3, 64, 4, 6, dtype=torch.bfloat16)
    g = torch.Generator().manual_seed(2)
    fused = torch.randn(2, 21, 13, 64, generator=g).bfloat16()
    ids, start = [0, 2, 3], [0, 5, 5, 20]
    m.reserve(ids, [9, 0, 30])
    m.append(ids, start, fused[:, :, 7:10], fused[:, :, 10:13], None)
    m.append(ids, start, fused[1, :, 4:7], fused[1, :, 7:10], 1)
    d = fused.cuda()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        seqs = i32(ids)
        c.reserve(i32([9, 0, 30]), seqs)
        c.append(d[:, :, 7:10], d[:, :, 10:13], i32(start), seqs=seqs)
        c.append(d[1, :, 4:7], d[1, :, 7:10], i32(start), layer=1, seqs=seqs)
    torch.cuda.current_stream().wait_stream(s)
    same(c, m)


@pytest.mark.gpu
def test_copy_pages_between_caches():
    c, m = pair(3, 20, 16, 3, 72, 4, 6, dtype=torch.bfloat16)
    o, _ = pair(3, 9, 16, 3, 72, 2, 3, dtype=torch.bfloat16)
    want = [o.k.clone(), o.v.clone()]
    src, dst = [3, 3, 0, 19], [8, 1, 2, 0]
    for w, pool in zip(want, (c.k, c.v)):
        w[:, dst] = pool[:, src]
    c.copy(i32(src), i32(dst), to=o)
    assert torch.equal(o.k, want[0]) and torch.equal(o.v, want[1])
    c.copy(i32([1, 2]), i32([5, 20]))
    assert mls.mls_get_status() == BAD
    assert torch.equal(c.k[:, 5], c.k[:, 1])
    with pytest.raises(mls.MLSError):
        c.copy(i32([1]), i32([1]), to=mls.PagedCache(3, 9, 8, 3, 72, 2, 3))


@pytest.mark.gpu
def test_a_captured_round_replays():
    """A round's calls in one graph, replayed on a state that changes from one to the next."""
    c, m = pair(2, 64, 16, 2, 64, 6, 8, dtype=torch.bfloat16)
    g = torch.Generator().manual_seed(3)
    m.reserve([0, 1], [40, 16])
    m.compact([0, 1], [40, 16], None)
    c.reserve(i32([40, 16]))
    c.compact(i32([40, 16]))
    kids, src, count, start = i32([3, 4]), i32([0, 1]), i32([6, 6]), i32([0, 6, 12])
    keep, path = i32([3, 2]), i32([[0, 2, 5], [0, 4, -1]])
    k, v = (torch.randn(2, 12, 2, 64, generator=g).bfloat16() for _ in range(2))
    kd, vd = k.cuda(), v.cuda()

    def device():
        c.free(kids)
        c.fork(src, kids)
        c.reserve(count, kids)
        c.append(kd, vd, start, seqs=kids)
        c.compact(keep, path, kids)
        c.reserve(i_one, first)
        c.compact(i_one, None, first)

    def model():
        m.free([3, 4])
        m.fork([0, 1], [3, 4])
        m.reserve([3, 4], [6, 6])
        m.append([3, 4], [0, 6, 12], k, v, None)
        m.compact([3, 4], [3, 2], [[0, 2, 5], [0, 4, -1]])
        m.reserve([0], [1])
        m.compact([0], [1], None)

    i_one, first = i32([1]), i32([0])
    device()
    model()
    same(c, m)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s), torch.cuda.graph(graph, stream=s):
        device()
    for _ in range(12):
        graph.replay()
        torch.cuda.synchronize()
        model()
        same(c, m)


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes and 2^31 values a tensor: what lies at its end."""
    pages = 4300
    c = mls.PagedCache(4, pages, 256, 4, 128, 2, 8)
    assert c.k.numel() > 1 << 31
    c.refs[:pages - 3] = 1
    c.free_bits.zero_()
    for p in range(pages - 3, pages):
        c.free_bits[p // 32] |= (1 << (p % 32)) - (1 << 32 if p % 32 == 31 else 0)
    n = 600
    c.reserve(i32([n]))
    assert c.table[0, :3].tolist() == [pages - 3, pages - 2, pages - 1]
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn(4, n, 4, 128, generator=g, device="cuda").bfloat16() for _ in range(2))
    c.append(k, v, i32([0, n]))
    path = list(range(0, n, 3))
    c.compact(i32([len(path)]), i32([path]))
    for pool, new in ((c.k, k), (c.v, v)):
        got = pool[:, pages - 3].permute(0, 2, 1, 3)[:, :len(path)]
        assert torch.equal(got, new[:, path])
    assert c.held[0] == 1 and mls.mls_get_status() == 0


def test_refusals():
    """What the host can see is refused before any launch (no GPU)."""
    L, P = B.lib(), 0x1000
    p = ctypes.c_void_p(P)

    def cache(layers=2, pages=10, ps=16, heads=2, dim=64, dtype=B.MLS_BF16, seqs=4, most=4, k=P, table=P):
        return B.mls_cache(layers, pages, ps, heads, dim, dtype, seqs, most, k, P, table, P, P, P, P)

    def reserve(n=2, count=p, ids=None, **kw):
        return L.mls_cache_reserve(ctypes.byref(cache(**kw)), n, ids, count, None)

    for kw in (dict(layers=0), dict(pages=0), dict(heads=0), dict(dim=0), dict(dtype=7), dict(seqs=0), dict(most=0),
               dict(k=None), dict(table=None), dict(n=-1), dict(n=5), dict(count=None)):
        assert reserve(**kw) == B.MLS_ERR_ARG, kw
    for kw in (dict(ps=12), dict(ps=4), dict(ps=512), dict(dim=60), dict(pages=(1 << 26) + 1), dict(most=(1 << 20) + 1),
               dict(heads=1 << 28), dict(seqs=20000, n=9000)):
        assert reserve(**kw) == B.MLS_ERR_UNSUPPORTED, kw
    for kw in (dict(k=P + 8), dict(table=P + 2), dict(count=ctypes.c_void_p(P + 1)), dict(ids=ctypes.c_void_p(P + 2))):
        assert reserve(**kw) == B.MLS_ERR_ALIGN, kw
    assert reserve(n=0, count=None) == B.MLS_OK
    c = cache()
    r = ctypes.byref(c)

    def append(layer=0, n=2, N=5, k=p, ld=128, lld=1000, start=p):
        return L.mls_cache_append(r, layer, n, None, start, N, k, p, ld, lld, None)

    assert append(layer=2) == append(layer=-2) == append(N=-1) == append(k=None) == append(start=None) == B.MLS_ERR_ARG
    assert append(ld=127) == append(ld=1 << 50) == append(layer=-1, lld=-8) == B.MLS_ERR_ARG
    assert append(ld=132) == append(layer=-1, lld=1001) == append(k=ctypes.c_void_p(P + 8)) == B.MLS_ERR_ALIGN
    assert append(N=0, k=None) == append(n=0) == B.MLS_OK
    assert L.mls_cache_compact(r, 2, None, None, None, 0, None) == B.MLS_ERR_ARG
    assert L.mls_cache_compact(r, 2, None, p, p, 0, None) == B.MLS_ERR_ARG
    size = B.mls_cache_workspace_size(c)
    assert size >= 2 * 4 * 4
    assert L.mls_cache_fork(r, 2, p, p, None, size, None) == B.MLS_ERR_WORKSPACE
    assert L.mls_cache_fork(r, 2, p, p, p, size - 1, None) == B.MLS_ERR_WORKSPACE
    assert L.mls_cache_fork(r, 2, None, p, p, size, None) == B.MLS_ERR_ARG
    assert L.mls_cache_free(r, 5, None, None) == B.MLS_ERR_ARG
    assert L.mls_cache_copy(r, ctypes.byref(cache(ps=32)), 1, p, p, None) == B.MLS_ERR_ARG
    assert L.mls_cache_reset(None, None) == B.MLS_ERR_ARG
    assert B.mls_cache_workspace_size(cache(ps=12)) == 0
    assert B.mls_strerror(NONE) != "unknown code"
    with pytest.raises(TypeError):
        mls.PagedCache(1, 4, 16, 1, 64, 1, 4, dtype=torch.float16, device="cpu")
    with pytest.raises(ValueError):
        mls.PagedCache(1, 4, 16, 1, 64, 1, 4, device="cpu")
    with pytest.raises(ValueError):
        mls.PagedCache(1, 4, 16, 0, 64, 1, 4, device="cpu")
