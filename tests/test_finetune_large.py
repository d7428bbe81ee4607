"""Offsets that pass 32 bits: tensors of more than 2^31 values.  The far end of each large
call has to equal, bit for bit, a small call on the same values (every row, token and
32-value group is computed alike wherever it lies)."""
import math

import pytest
import torch

import paper_2608_09703_gb300 as mls

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 120 << 30:
        pytest.skip("needs 120 GB of free device memory")
    yield
    torch.cuda.empty_cache()


def test_layer_norm():
    T, d = 530000, 4104
    assert T * d > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(T, d, dtype=torch.bfloat16, device="cuda").normal_(0.3, 1.0, generator=g)
    dy = torch.empty_like(x).normal_(0.0, 1.0, generator=g)
    w = torch.empty(d, dtype=torch.bfloat16, device="cuda").normal_(1.0, 0.1, generator=g)
    op = mls.LayerNorm(T, d)
    op.forward(x, w, w)
    op.backward(x, dy, w)
    n = 50
    small = mls.LayerNorm(n, d)
    small.forward(x[-n:].contiguous(), w, w)
    small.backward(x[-n:].contiguous(), dy[-n:].contiguous(), w)
    for a, b in ((op.y, small.y), (op.mean, small.mean), (op.rstd, small.rstd), (op.dx, small.dx)):
        assert torch.equal(a[-n:], b)
    want = sum(dy[i:i + 10000].double().sum(0) for i in range(0, T, 10000))
    # 530000 terms of fp32 sums, some 250 rows in a chain: (250 + 152 + 16) 2^-24 of their sizes
    size = sum(dy[i:i + 10000].double().abs().sum(0) for i in range(0, T, 10000))
    assert bool(((op.dbias.double() - want).abs() <= 4000 * 2.0 ** -24 * size).all())


def test_policy_loss():
    T, M = 560000000, 4
    assert T * M > 1 << 31
    logp = torch.zeros(M, T, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    logp[3, -5000:].normal_(-1.0, 0.5, generator=g)
    adv, y = torch.ones(T, device="cuda"), torch.full((T,), -1, dtype=torch.int32, device="cuda")
    y[-5000:] = 7
    old = torch.zeros(M, T, device="cuda")
    prob = mls.PolicyProblem(T, 100, M=M)
    ws = torch.empty(mls.mls_policy_workspace_size(prob), dtype=torch.uint8, device="cuda")
    loss, diag, dlogp = torch.empty(1, device="cuda"), torch.empty(3, M, device="cuda"), torch.full_like(logp, 5.0)
    mls.mls_policy_loss(prob, logp, old, None, adv, y, None, 1.0, loss, None, diag, dlogp, ws)
    small = mls.PolicyLoss(5000, 100, M=M)
    small(logp[:, -5000:].contiguous(), old[:, -5000:].contiguous(), adv[-5000:], y[-5000:])
    assert torch.equal(dlogp[:, -5000:], small.dlogp)
    assert not any(dlogp[m, :-5000].any() for m in range(M))
    assert abs(loss.item() - small.loss.item()) <= 32 * 2.0 ** -24 * float(small.tok_loss.abs().sum()) / 5000


def test_grad_clip():
    n = (1 << 31) + 12345
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-1], g[1 << 31], g[5] = 3.0, 4.0, 12.0
    norm, c = mls.GradClip([g[1:]])(6.5).tolist()
    assert norm == 13.0 and c == pytest.approx(0.5, rel=1e-6)
    assert (g[-1].item(), g[1 << 31].item(), g[5].item()) == (1.5, 2.0, 6.0)
    assert math.isclose(float(g.float().sum()), 9.5)


def test_log_probabilities():
    # dL/dz of one group and dW pass 2^31 values
    T, d, V = 17000, 8192, 270000
    assert T * 131072 > 1 << 31 and V * d > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(3)
    H = torch.empty(T, d, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=g)
    W = torch.empty(V, d, dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.02, generator=g)
    y = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    y[-3:] = torch.tensor([V - 1, 5, V - 2], dtype=torch.int32, device="cuda")
    dl = torch.ones(1, T, device="cuda")
    op = mls.HeadLogp((d,), T, V, vocab_group=135168)
    op.forward([H], [W], y)
    dH, dW = op.backward([H], [W], y, dl)
    rows = H[-3:].double() @ W.double().T
    lse = torch.logsumexp(rows, 1)
    p = torch.exp(rows - lse[:, None])
    want = rows.gather(1, y[-3:].long()[:, None])[:, 0] - lse
    assert bool(((op.logp[0, -3:].double() - want).abs() <= 2e-4).all())  # 2 d 2^-24 of 130 at most
    G = -p
    G[torch.arange(3), y[-3:].long()] += 1
    far = G.T[-64:] @ H[-3:].double()
    assert float((dW[0][-64:].double() - far).norm() / far.norm()) < 2.0 ** -7
    near = G @ W.double()
    assert float((dH[0][-3:].double() - near).norm() / near.norm()) < 2.0 ** -7
    assert not dH[0][:-3].any()
    assert mls.mls_get_status() == 0
