"""The number of sequences that a policy loss takes, refused by the host beyond."""
import ctypes

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from paper_2608_09703_gb300 import build as mbuild


@pytest.mark.parametrize("agg", ["token", "seq", "sum"])
def test_more_sequences_than_32_bits_can_step_through(agg):
    mbuild.build()
    p = 0x1000

    def call(n, size=1 << 40):
        prob = mls.PolicyProblem(100, 1000, B=n, agg=agg)
        return B.mls_policy_workspace_size(prob), B.lib().mls_policy_loss(
            prob.ref(), p, p, p, p, p, p, 1.0, p, p, p, 0x2000, 0x10000, size, None)

    for n in (B.MLS_POLICY_MAX_SEQS + 1, (1 << 31) - 256, (1 << 31) - 30, (1 << 31) - 2, (1 << 31) - 1):
        assert call(n) == (0, B.MLS_ERR_UNSUPPORTED)
    # the last one accepted gets as far as its pointers
    prob = mls.PolicyProblem(100, 1000, B=B.MLS_POLICY_MAX_SEQS, agg=agg)
    assert B.mls_policy_workspace_size(prob) > 0
    assert B.lib().mls_policy_loss(prob.ref(), ctypes.c_void_p(p + 2), p, p, p, p, p, 1.0, p, p, p, 0x2000, 0x10000,
                                   1 << 40, None) == B.MLS_ERR_ALIGN


def step_32(lo, hi):
    """The search's step over [lo, hi] as the kernel forms it, in wrapping 32 bits."""
    v = (hi - lo + 31 + (1 << 31)) % (1 << 32) - (1 << 31)
    return int(v / 32)


def test_steps_stay_positive_up_to_the_limit():
    assert step_32(0, (1 << 31) - 30) < 0  # what the limit keeps away
    for n in (1, 2, 33, 1 << 20, B.MLS_POLICY_MAX_SEQS):
        lo, hi = 0, n - 1
        while lo < hi:  # the path that moves furthest up: every candidate starts at or before the token
            step = step_32(lo, hi)
            assert step > 0 and lo + 32 * step + step < 1 << 31
            k = min(32, (hi - lo) // step)
            lo, hi = lo + k * step, min(hi, lo + k * step + step - 1)
        assert n + 1024 < 1 << 31  # the check of the offsets, a block's threads a step


@pytest.mark.gpu
@pytest.mark.parametrize("T,n", [(3, 7), (3, 5000), (4096, 4096), (5000, 3), (5000, 70000), (70001, 1024), (70001, 300000)])
def test_any_bad_offset_is_reported(T, n):
    """Every offset is looked at, by whichever block: one alone that is out of order or range."""
    g = torch.Generator(device="cuda").manual_seed(n)
    start = torch.randint(0, T + 1, (n + 1,), generator=g, device="cuda").sort().values.int()
    logp, adv = torch.zeros(1, T, device="cuda"), torch.ones(T, device="cuda")
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    op = mls.PolicyLoss(T, 10, B=n)
    op(logp, logp, adv, y, seq_start=start)
    assert mls.mls_get_status() == 0
    for b in sorted({0, 1, n // 3, n // 2, n - 1, n, min(n, 1023), min(n, 1024), min(n, 4095), min(n, 4096)}):
        for v in (-1, T + 1):
            bad = start.clone()
            bad[b] = v
            op(logp, logp, adv, y, seq_start=bad)
            assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ, (b, v)
    if n > 1:
        bad = torch.arange(n + 1, device="cuda").clamp(max=T).int()
        bad[n // 2], bad[n // 2 - 1] = 0, max(1, min(T, n // 2 - 1))
        if n // 2 > 1:
            op(logp, logp, adv, y, seq_start=bad)
            assert mls.mls_get_status() == B.MLS_STATUS_BAD_SEQ


@pytest.mark.gpu
@pytest.mark.parametrize("T", [700, 70001])
@pytest.mark.parametrize("low,high", [(1.0, float("inf")), (0.2, float("inf")), (3.0, 0.28)])
def test_bounds_that_are_none(T, low, high):
    """No ratio is past an infinite bound, an infinite ratio neither."""
    g = torch.Generator(device="cuda").manual_seed(T)
    old = torch.randn(1, T, generator=g, device="cuda")
    logp = old + 2 * torch.randn(1, T, generator=g, device="cuda")
    logp[0, :3], old[0, :3] = torch.tensor([3e38, -3e38, 100.0]), torch.tensor([-3e38, 3e38, 0.0])
    adv = torch.randn(T, generator=g, device="cuda")
    adv[:3] = torch.tensor([1.0, -1.0, 1.0])
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    op = mls.PolicyLoss(T, 10, clip_low=low, clip_high=high, agg="sum")
    op(logp, old, adv, y)
    r = torch.exp(logp.double() - old.double())[0]
    hi, lo = 1 + float(torch.tensor(high)), max(0.0, 1 - float(torch.tensor(low)))
    stop = ((adv > 0) & (r > hi)) | ((adv < 0) & (r < lo))
    assert torch.equal(op.dlogp[0] == 0, stop | (r.float() == 0))
    assert float(op.diag[2, 0]) == float(stop.sum())
    on = ~stop & torch.isfinite(r.float()) & (r > 1e-30)
    want = -r * adv.double()
    tol = 2.0 ** -24 * ((logp - old).abs()[0].double() + 16)
    assert bool(((op.dlogp[0].double() - want).abs() <= tol * want.abs())[on].all())
    assert mls.mls_get_status() == 0
