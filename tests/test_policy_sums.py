"""The loss and the diagnostics of a short batch, as sums: ratios of 1 and weights that are powers of
two make every term exact, so the sum's own error is all there is, on terms that cancel.

Tolerances, u = 2^-24: sums in two words keep 2^-44 of the terms' sizes (each of at most a dozen
steps rounds the second word, 2^-48 of the first), and the result is rounded once, the loss of a
sub-model's weight and its sum with the others' again."""
import pytest
import torch

import paper_2608_09703_gb300 as mls

U = 2.0 ** -24


@pytest.mark.gpu
@pytest.mark.parametrize("T", [1, 2, 33, 256, 512, 1000, 1024])
@pytest.mark.parametrize("M", [1, 2, 4])
@pytest.mark.parametrize("agg", ["token", "seq", "sum"])
def test_terms_that_cancel(T, M, agg):
    n = 1 << (T.bit_length() - 1)  # as many tokens count
    for seed in range(8):
        g = torch.Generator(device="cuda").manual_seed(seed)
        logp = -torch.empty(M, T, device="cuda").exponential_(1.0, generator=g)
        adv = torch.randn(T, generator=g, device="cuda") * torch.where(torch.arange(T, device="cuda") % 3 == 0, 100.0, 1.0)
        adv[:n] -= adv[:n].mean()
        y = torch.where(torch.arange(T, device="cuda") < n, 1, -1).int()
        start = torch.tensor([0, n // 2, n], dtype=torch.int32, device="cuda") if agg == "seq" and n > 1 else \
            torch.tensor([0, n], dtype=torch.int32, device="cuda")
        op = mls.PolicyLoss(T, 10, M=M, B=len(start) - 1, agg=agg)
        op(logp, logp, adv, y, seq_start=start)
        weight = 1.0 if agg == "sum" else 1.0 / n
        want, size = -float(adv[:n].double().sum()) * weight, float(adv[:n].double().abs().sum()) * weight
        bound = U * abs(want) + 2.0 ** -44 * size
        assert bool(((op.diag[0].double() - want).abs() <= bound).all()), (op.diag[0].tolist(), want, size)
        assert abs(float(op.loss) - M * want) <= U * abs(M * want) + M * 2.0 ** -44 * size
