"""Rounds of speculative decoding with a shared cache as they are used: prompts read in as chains, samples forked
from them, then round after round reserve, append, tree attention, tree verification, compact.  Keys and values
of a token are functions of the token, its position and the layer, so what the cache holds at the end says
whether every call did its part: the accepted tokens, in order, and nothing else."""
import pytest
import torch

import paper_2608_09703_gb300 as mls
from test_tree_attention import check

V, LAYERS, KV, HEADS, DIM, PAGE, WIDTH = 499, 3, 2, 8, 64, 16, 3


class Rounds:
    """S prompts, two samples of each, trees of n nodes a round."""

    def __init__(self, dtype, S=4, n=9, rounds=6, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.S, self.B, self.n, self.rounds = dtype, S, 2 * S, n, rounds
        self.k_of, self.v_of = (torch.randn(LAYERS, V, KV, DIM, generator=g).to(dtype).cuda() for _ in range(2))
        self.k_at, self.v_at = (torch.randn(LAYERS, 512, KV, 1, generator=g).to(dtype).cuda() for _ in range(2))
        self.prompts = [torch.randint(0, V, (int(torch.randint(1, 60, (1,), generator=g)),), generator=g) for _ in range(S)]
        self.draft = torch.softmax(torch.randn(V, V, generator=g) * 1.5, 1).cuda()       # of what follows a token
        self.target = torch.softmax(torch.log(self.draft) + torch.randn(V, V, generator=g).cuda() * 0.5, 1)
        self.q = (torch.randn(rounds, self.B * n, HEADS, DIM, generator=g) * 2).to(dtype).cuda()
        self.u = torch.rand(rounds, self.B * n, 2, generator=g).cuda()
        # a tree's shape: the same for all, so that shapes do not change from round to round
        up = [-1] + [max(0, i - 1 - int(torch.randint(0, min(i, WIDTH), (1,), generator=g))) for i in range(1, n)]
        self.up = torch.tensor(up)
        self.depth = torch.zeros(n, dtype=torch.long)
        for i in range(1, n):
            self.depth[i] = self.depth[up[i]] + 1
        self.up, self.depth = self.up.cuda(), self.depth.cuda()
        self.pick = torch.rand(rounds, self.B, n, generator=g).cuda()
        self.parents = self.up.int().repeat(self.B)
        self.start = torch.arange(0, self.B * n + 1, n, dtype=torch.int32).cuda()

    def kv(self, tokens, at):
        """Keys and values [LAYERS, N, KV, DIM] of tokens at positions."""
        return self.k_of[:, tokens] + self.k_at[:, at], self.v_of[:, tokens] + self.v_at[:, at]

    def begin(self):
        most = 512 // PAGE
        self.cache = c = mls.PagedCache(LAYERS, 3 * self.B * most, PAGE, KV, DIM, self.S + self.B, most, dtype=self.dtype)
        lens = [len(t) for t in self.prompts]
        N = sum(lens)
        count = torch.tensor(lens, dtype=torch.int32).cuda()
        rows = torch.arange(self.S, dtype=torch.int32).cuda()
        start = torch.tensor([0] + lens).cumsum(0).int().cuda()
        tokens = torch.cat(self.prompts).cuda()
        at = torch.cat([torch.arange(n) for n in lens]).cuda()
        k, v = self.kv(tokens, at)
        c.reserve(count, seqs=rows)
        c.append(k, v, start, seqs=rows)
        chain = mls.TreeAttention(c, self.S, N, HEADS)
        g = torch.Generator().manual_seed(1)
        q = (torch.randn(N, HEADS, DIM, generator=g) * 2).to(self.dtype).cuda()
        for layer in range(LAYERS):
            out, lse = chain(q, start, None, layer, seqs=rows)
            x = dict(news=lens, lens=[0] * self.S, start=start.cpu(), parents=None, q=q.cpu(), dtype=self.dtype,
                     k=c.k[layer:layer + 1].cpu(), keys=[t.cpu() for t in k[layer].split(lens)],
                     values=[t.cpu() for t in v[layer].split(lens)])
            check(x, out.cpu(), lse.cpu(), chain.scale)
        c.compact(count, seqs=rows)
        # two samples of each prompt
        self.rows = torch.arange(self.S, self.S + self.B, dtype=torch.int32).cuda()
        c.fork(rows.repeat_interleave(2), self.rows)
        self.attend = mls.TreeAttention(c, self.B, self.B * self.n, HEADS)
        self.verify = mls.TreeVerify(self.B, self.B * self.n, V, max_path=self.n)
        self.last = torch.stack([t[-1] for t in self.prompts]).repeat_interleave(2).cuda()  # follows what is cached
        self.fresh = torch.zeros_like(self.last)
        self.seen = []
        self.count = torch.full((self.B,), self.n, dtype=torch.int32).cuda()

    def draw(self, pick):
        """The tree's tokens: node 0 the last one accepted, the others drawn from the draft's rows."""
        tokens = torch.zeros(self.B, self.n, dtype=torch.long, device="cuda")
        tokens[:, 0] = self.last
        for i in range(1, self.n):
            rows = self.draft[tokens[:, self.up[i]]].double().cumsum(1)
            tokens[:, i] = torch.searchsorted(rows, pick[:, i:i + 1].double() * rows[:, -1:], right=True)[:, 0].clamp(max=V - 1)
        return tokens

    def calls(self, k, v, q, target, draft, tokens, u):
        """What a round launches."""
        c = self.cache
        c.reserve(self.count, seqs=self.rows)
        out = []
        for layer in range(LAYERS):
            c.append(k[layer], v[layer], self.start, layer=layer, seqs=self.rows)
            o, lse = self.attend(q, self.start, self.parents, layer, seqs=self.rows)
            out.append((o.clone(), lse.clone()))
        n_path, path, token = self.verify(target, tokens, self.parents, self.start, u, draft=draft)
        c.compact(n_path, path=path, seqs=self.rows)
        return out, n_path, path, token

    def inputs(self, r):
        tokens = self.draw(self.pick[r])
        lens = self.cache.len[self.S:].long()
        k, v = self.kv(tokens.flatten(), (lens[:, None] + self.depth).flatten())
        flat = tokens.flatten()
        return dict(k=k, v=v, q=self.q[r], target=self.target[flat], draft=self.draft[flat], tokens=flat.int(), u=self.u[r])


def play(rounds, graph):
    """All rounds; returns the accepted tokens of every sample, and every round's outputs."""
    s = rounds
    s.begin()
    accepted = [[] for _ in range(s.B)]
    log, captured, held = [], None, None
    for r in range(s.rounds):
        x = s.inputs(r)
        lens = s.cache.len[s.S:].tolist()
        before = [t[s.S:].clone() for t in (s.cache.table, s.cache.len)]
        if graph and r == 1:  # the second round is captured, and replayed from then on
            held = {a: b.clone() for a, b in x.items()}
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.stream(side), torch.cuda.graph(captured, stream=side):
                result = s.calls(**held)
            torch.cuda.current_stream().wait_stream(side)
        if captured:
            for a, b in x.items():
                held[a].copy_(b)
            captured.replay()
        else:
            result = s.calls(**x)
        torch.cuda.synchronize()
        assert mls.mls_get_status() == 0
        out, n_path, path, token = result
        log.append(([(o.clone(), lse.clone()) for o, lse in out], n_path.clone(), path.clone(), token.clone(), x, before, lens))
        s.last = token.long().clone()
        tokens = x["tokens"].view(s.B, s.n)
        for b in range(s.B):
            accepted[b] += [int(tokens[b, j]) for j in path[b, :int(n_path[b])]]
    return accepted, log


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rounds(dtype):
    s = Rounds(dtype)
    accepted, log = play(s, False)
    c = s.cache
    assert sum(len(a) for a in accepted) > s.rounds * s.B + 5  # some drafts were accepted, some trees refused
    assert any(int((x[1] == 1).sum()) for x in log)
    # what the cache holds: each prompt's tokens and the accepted ones, at their positions
    for b in range(s.B):
        tokens = torch.cat([s.prompts[b // 2], torch.tensor(accepted[b])]).cuda()
        n = len(tokens)
        assert int(c.len[s.S + b]) == n and int(c.held[s.S + b]) == -(-n // PAGE)
        k, v = s.kv(tokens, torch.arange(n, device="cuda"))
        pages = c.table[s.S + b, :-(-n // PAGE)].long()
        for have, want in ((c.k, k), (c.v, v)):
            have = have[:, pages].permute(0, 1, 3, 2, 4).reshape(LAYERS, -1, KV, DIM)[:, :n]
            assert torch.equal(have, want), b
    # pages: whole ones of a prompt have three owners, others one
    owners = torch.bincount(c.table[c.table >= 0].long(), minlength=c.refs.numel())
    assert torch.equal(owners.int(), c.refs)
    for b, t in enumerate(s.prompts):
        assert (c.refs[c.table[b, :len(t) // PAGE].long()] == 3).all()
    # every round's attention, layer by layer, against the definition
    have = [list(t.tolist()) for t in s.prompts for _ in range(2)]
    for out, n_path, path, token, x, _, lens in log:
        tokens = x["tokens"].view(s.B, s.n)
        for layer, (o, lse) in enumerate(out):
            keys, values = [], []
            for b in range(s.B):
                k, v = s.kv(torch.tensor(have[b]).cuda(), torch.arange(len(have[b]), device="cuda"))
                new = slice(b * s.n, (b + 1) * s.n)
                keys.append(torch.cat([k[layer], x["k"][layer, new]]).cpu())
                values.append(torch.cat([v[layer], x["v"][layer, new]]).cpu())
            y = dict(news=[s.n] * s.B, lens=lens, start=s.start.cpu(), parents=s.parents.cpu(), q=x["q"].cpu(), dtype=dtype,
                     k=c.k[:1].cpu(), keys=keys, values=values)
            check(y, o.cpu(), lse.cpu(), s.attend.scale)
        for b in range(s.B):
            have[b] += [int(tokens[b, j]) for j in path[b, :int(n_path[b])]]
    # and back: everything is free
    c.free()
    assert int(c.refs.abs().sum()) == 0 and int(c.len.sum()) == 0
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_captured_rounds(dtype):
    """Rounds replayed from one graph accept the same tokens and leave the same cache."""
    a, b = Rounds(dtype, seed=3), Rounds(dtype, seed=3)
    one, log1 = play(a, False)
    two, log2 = play(b, True)
    assert one == two
    for x, y in zip(log1, log2):
        for (o1, l1), (o2, l2) in zip(x[0], y[0]):
            assert torch.equal(o1, o2) and torch.equal(l1, l2)
        assert all(torch.equal(x[i], y[i]) for i in (1, 2, 3))
    for name in ("table", "len", "held", "refs", "free_bits"):
        assert torch.equal(getattr(a.cache, name), getattr(b.cache, name)), name
