"""The log-probabilities read none of the loss's fields of a problem, whatever they hold."""
import ctypes

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from paper_2608_09703_gb300 import build as mbuild

NAN = float("nan")
FIELDS = [dict(teacher=-1), dict(teacher=7), dict(alpha=-3.0), dict(alpha=NAN), dict(w=[NAN, 1.0]),
          dict(teacher=1 << 30, alpha=float("inf"), w=[float("inf")] * 2)]


@pytest.mark.parametrize("fields", FIELDS)
def test_not_refused(fields):
    mbuild.build()
    L, p, odd = B.lib(), 0x1000, 0x1008
    plain, prob = mls.Problem((64, 72), 10, 100), mls.Problem((64, 72), 10, 100, **fields)
    assert B.mls_logp_workspace_size(prob) == B.mls_logp_workspace_size(plain) > 0

    def arr(v, k=2):
        return (ctypes.c_void_p * k)(v, v + 0x1000)

    # as far as its pointers: one off its boundary
    ws = (0x10000, 1 << 40, None)
    assert L.mls_head_logp_fwd(prob.ref(), arr(odd), arr(p), p, p, p, *ws) == B.MLS_ERR_ALIGN
    assert L.mls_head_logp_fwd_peak(prob.ref(), arr(odd), arr(p), p, p, p, p, *ws) == B.MLS_ERR_ALIGN
    assert L.mls_head_logp_bwd(prob.ref(), arr(odd), arr(p), p, p, p, arr(p), arr(p), *ws) == B.MLS_ERR_ALIGN
    assert L.mls_head_logp_bwd_peak(prob.ref(), arr(odd), arr(p), p, p, p, p, arr(p), arr(p), *ws) == B.MLS_ERR_ALIGN
    # the loss still reads them
    assert B.mls_workspace_size(prob) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 2, 4])
def test_same_results(M):
    d, T, V = (64, 72, 136, 8)[:M], 70, 700
    g = torch.Generator(device="cuda").manual_seed(M)
    H = [torch.randn(T, dm, generator=g, device="cuda").bfloat16() for dm in d]
    W = [torch.randn(V, dm, generator=g, device="cuda").bfloat16() for dm in d]
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    dl = torch.randn(M, T, generator=g, device="cuda")
    out = []
    for fields in (dict(), dict(teacher=1 << 30, alpha=NAN, w=[NAN] * M)):
        op = mls.HeadLogp(d, T, V)
        op.prob = mls.Problem(d, T, V, **fields)
        op.forward(H, W, y)
        op.backward(H, W, y, dl)
        out.append([op.logp, op.lse] + op.dH + op.dW)
    assert all(torch.equal(a, b) for a, b in zip(*out))
    assert mls.mls_get_status() == 0
