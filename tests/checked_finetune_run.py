"""Child process of tests/test_checked_finetune.py: runs the fine-tuning operators of the
library that the environment selects (MLS_CHECKED=1: the checked build) on small ragged
cases and saves the outputs and the status words to an .npz."""
import sys

import numpy as np
import torch

import paper_2608_09703_gb300 as mls


def main(path):
    out, g = {}, torch.Generator(device="cuda").manual_seed(5)

    def r(*s):
        return torch.randn(*s, generator=g, device="cuda")

    def keep(tag, **tensors):
        torch.cuda.synchronize()
        out["status_" + tag] = np.array(mls.mls_get_status())
        for k, t in tensors.items():
            if t is not None:
                out[f"{tag}_{k}"] = t.float().cpu().numpy()

    # two vocabulary groups, split reductions, wide units, extra pairs, four sub-models
    for tag, T, d, V, group in (("g", 300, (64, 128, 192), 1000, 512), ("s", 1100, (320, 1008), 33000, 0),
                                ("w", 2700, (264, 776), 33000, 0), ("x", 1290, (72, 64, 80), 25523, 0),
                                ("m", 500, (64, 8, 64, 192), 2000, 0)):
        H = [r(T, dm).bfloat16() for dm in d]
        W = [(0.1 * r(V, dm)).bfloat16() for dm in d]
        y = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
        op = mls.HeadLogp(d, T, V, tau=0.9, vocab_group=group)
        op.forward(H, W, y)
        dH, dW = op.backward(H, W, y, r(len(d), T))
        keep("logp_" + tag, logp=op.logp, lse=op.lse, **{f"dH{m}": t for m, t in enumerate(dH)},
             **{f"dW{m}": t for m, t in enumerate(dW)})
    for T, d in ((33, 72), (130, 2056), (70, 9000), (20, 16640)):
        x, gain, bias, dy = r(T, d).bfloat16(), r(d).bfloat16(), r(d).bfloat16(), r(T, d).bfloat16()
        op = mls.LayerNorm(T, d)
        y = op.forward(x, gain, bias)
        op.backward(x, dy, gain)
        keep(f"norm{d}", y=y, mean=op.mean, rstd=op.rstd, dx=op.dx, dgain=op.dgain, dbias=op.dbias)
    for T, n in ((700, 5), (9000, 60), (40000, 3)):
        logp = -r(2, T).abs()
        start = torch.randint(0, T + 1, (n + 1,), generator=g, device="cuda").sort().values.to(torch.int32)
        y = torch.randint(-2, 9, (T,), generator=g, device="cuda", dtype=torch.int32)
        for agg in ("token", "seq", "sum"):
            op = mls.PolicyLoss(T, 9, M=2, B=n, beta=0.1, agg=agg, adv_per_seq=True)
            op(logp, logp + 0.3 * r(2, T), r(n), y, ref_logp=logp + 0.2 * r(2, T), seq_start=start)
            keep(f"policy{T}{agg}", loss=op.loss, tok=op.tok_loss, diag=op.diag, dlogp=op.dlogp)
    grads = [r(n) for n in (1, 9001, 77)] + [r(n).bfloat16() for n in (5, 30000)]
    stats = mls.GradClip(grads)(1.0)
    keep("clip", stats=stats, **{f"g{i}": t for i, t in enumerate(grads)})
    np.savez(path, **out)


if __name__ == "__main__":
    main(sys.argv[1])
