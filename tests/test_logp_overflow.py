"""Tokens without a gradient whose logits overflow: rows of finite values that are past any
product's range (memory that padding left as it was) reach no gradient."""
import pytest
import torch

import paper_2608_09703_gb300 as mls

FAR = 3.0e38


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V,group", [(64, (64,), 300, 0), (300, (64, 136), 1025, 256), (40, (136,), 20000, 0)])
@pytest.mark.parametrize("mixed", [False, True])
def test_overflowed_logits_of_tokens_without_gradient(T, d, V, group, mixed):
    g = torch.Generator(device="cuda").manual_seed(T)
    H = [torch.randn(T, dm, generator=g, device="cuda").bfloat16() for dm in d]
    W = [torch.randn(V, dm, generator=g, device="cuda").bfloat16() for dm in d]
    y = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    dl = torch.randn(len(d), T, generator=g, device="cuda")
    left, none = torch.arange(T, device="cuda") % 7 == 3, torch.arange(T, device="cuda") % 7 == 5
    y[left] = -1
    dl[:, none] = 0.0
    off = left | none
    op = mls.HeadLogp(d, T, V, vocab_group=group)

    def grads(fill):
        h = [x.clone() for x in H]
        for x in h:
            x[off] = fill(x[off])
        op.forward(h, W, y)
        dH, dW = op.backward(h, W, y, dl)
        return [t.clone() for t in dH + dW], op.logp.clone()

    want, logp = grads(torch.zeros_like)
    # one sign: every logit infinite; both: infinities of both signs, and NaN where they meet
    got, same = grads(lambda x: torch.where(x > 0, FAR, -FAR).to(x.dtype) if mixed else torch.full_like(x, FAR))
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for m in range(len(d)):
        assert not got[m][off].any()
    assert torch.equal(same[:, ~off], logp[:, ~off]) and not same[:, left].any()
    assert mls.mls_get_status() == 0
