"""Child process of tests/test_checked_decoding.py: runs the decoding operators of the library that the environment
selects (MLS_CHECKED=1: the checked build) on small ragged cases and saves the outputs and the status words to an
.npz."""
import sys

import numpy as np
import torch

import paper_2608_09703_gb300 as mls


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def main(path):
    out, g = {}, torch.Generator(device="cuda").manual_seed(5)

    def r(*s):
        return torch.randn(*s, generator=g, device="cuda")

    def ints(lo, hi, *s):
        return torch.randint(lo, hi, s, generator=g, device="cuda", dtype=torch.int32)

    def keep(tag, **tensors):
        torch.cuda.synchronize()
        out["status_" + tag] = np.array(mls.mls_get_status())
        for k, t in tensors.items():
            out[f"{tag}_{k}"] = t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()

    def digest(t):
        """A sum over the bits of each page, by their places."""
        x = t.reshape(t.shape[0] * t.shape[1], -1).view(torch.int16).long()
        return (x * torch.arange(1, x.shape[1] + 1, device="cuda")).sum(1)

    # layers, kv heads, width, page, sequences, nodes of each, query heads, cached tokens up to
    for tag, dt, layers, kv, dim, page, S, n, heads, most in (
            ("a", torch.bfloat16, 2, 2, 128, 16, 5, 9, 8, 700), ("b", torch.bfloat16, 1, 1, 64, 8, 40, 3, 6, 130),
            ("c", torch.bfloat16, 3, 2, 72, 64, 2, 70, 12, 3000), ("d", torch.bfloat16, 1, 4, 128, 32, 64, 1, 4, 900),
            ("e", torch.float32, 2, 2, 128, 16, 5, 9, 8, 700), ("f", torch.float32, 1, 2, 40, 8, 30, 1, 4, 2000),
            ("g", torch.float32, 5, 1, 64, 128, 3, 150, 2, 300), ("h", torch.bfloat16, 1, 1, 96, 256, 2, 5, 160, 400)):
        width = (most + 2 * n) // page + 2
        c = mls.PagedCache(layers, S * width * 2, page, kv, dim, 2 * S, width, dtype=dt)
        c.k.copy_(r(*c.k.shape))
        c.v.copy_(r(*c.v.shape))
        lens = ints(0, most + 1, S)
        c.reserve(lens)
        c.compact(lens)
        kids = torch.arange(S, 2 * S, dtype=torch.int32, device="cuda")
        c.fork(ints(0, S, S), kids)
        more = ints(0, n + 1, S)
        more[0] = n
        start = torch.cat((i32([0]), more.cumsum(0).int()))
        N = S * n
        place = torch.cat([torch.arange(x) for x in more.tolist()] + [torch.zeros(N, dtype=torch.int64)])[:N].cuda()
        parents = (torch.rand(N, generator=g, device="cuda") * (place + 2)).int() - 2  # -2 .. place - 1
        for seqs in (kids, None):
            c.reserve(more, seqs)
            c.append(r(layers, N, kv, dim).to(dt), r(layers, N, kv, dim).to(dt), start, seqs=seqs)
            op = mls.TreeAttention(c, S, N, heads)
            for name, up in (("tree", parents), ("chain", None)):
                o, lse = op(r(N, heads, dim).to(dt), start, up, layers - 1, seqs)
                keep(f"{tag}{name}{seqs is None}", out=o, lse=lse)
            kept = 2 * torch.arange(n, dtype=torch.int32, device="cuda") + ints(0, 2, S, n)
            c.compact(more // 2, kept if seqs is None else None, seqs)
            keep(f"{tag}cache{seqs is None}", k=digest(c.k), v=digest(c.v), table=c.table, len=c.len, held=c.held, refs=c.refs,
                 bits=c.free_bits)
        c.copy(i32([0, 1]), i32([2, 3]))
        c.free(kids)
        keep(tag + "end", k=digest(c.k), table=c.table, refs=c.refs, bits=c.free_bits)
    for tag, S, n, V in (("a", 3, 7, 501), ("b", 70, 5, 33000), ("c", 2, 200, 9001), ("d", 1, 9, 128256)):
        p, q = (torch.softmax(2 * r(S * n, V), 1) for _ in range(2))
        parents = torch.stack([ints(max(-1, j - 4), j, S).clamp(min=0) if j else ints(-1, 0, S) for j in range(n)], 1).reshape(-1)
        tokens, u = ints(0, V, S * n), torch.rand(S * n, 2, generator=g, device="cuda")
        start = i32([n * i for i in range(S + 1)])
        for replace in (False, True):
            for draft in (q, None):
                op = mls.TreeVerify(S, S * n, V, max_path=n, replace=replace)
                a, b, c = op(p, tokens, parents, start, u, draft=draft)
                keep(f"verify{tag}{replace}{draft is None}", n=a, path=b, next=c)
    np.savez(path, **out)


if __name__ == "__main__":
    main(sys.argv[1])
