"""Hidden states wider than one accumulator's part of a reduction (1280 values at most).

Tolerances.  The tensor cores add 16 products at a time to an accumulator and truncate: each step
loses at most 2^-23 of what it holds then, and sums of positive terms grow evenly, so the n <= 80 steps
of a part lose at most n / 2 2^-23 of it, half of that on average, whatever the width.  (One accumulator
of all loses that for n = d / 16.)  The parts are added with rounding, 8 u for up to 8 of them."""
import pytest
import torch
from test_finetune_streams import STALL, _child
from test_logp import check, inputs

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B

U = 2.0 ** -24
STEPS = 1280 // 16


@pytest.mark.gpu
@pytest.mark.parametrize("d", [1024, 1032, 1280, 1288, 2048, 2056, 4096, 5128, 8192, 8200])
@pytest.mark.parametrize("tau", [1.0, 0.5])
def test_logits_of_positive_terms(d, tau):
    """One token in the vocabulary: its logsumexp is its logit."""
    T = 300
    g = torch.Generator(device="cuda").manual_seed(d)
    H = [(1 + torch.rand(T, d, generator=g, device="cuda")).bfloat16()]
    W = [((1 + torch.rand(1, d, generator=g, device="cuda")) / 16).bfloat16()]
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    op = mls.HeadLogp((d,), T, 1, tau=tau)
    logp = op.forward(H, W, y)
    assert not logp.any()
    want = (H[0].double() @ W[0].double().t())[:, 0] / tau
    rel = (op.lse[0].double() - want) / want
    n = min(STEPS, -(-d // 16))
    assert float(rel.abs().max()) <= n / 2 * 2.0 ** -23 + 16 * U
    assert abs(float(rel.mean())) <= n / 4 * 2.0 ** -23 + 16 * U


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,V,group", [(130, (1288, 2056), 1500, 0), (300, (1024, 1088, 4104), 1025, 256),
                                         (1, (8200,), 3000, 0), (513, (1296, 64), 2000, 512), (17, (64, 2048, 8, 1288), 700, 0),
                                         (2600, (1352,), 5003, 0)])
def test_against_the_definition(T, d, V, group):
    check(*inputs(d, T, V, seed=T + V), vocab_group=group)


@pytest.mark.gpu
def test_captured():
    """Replays of a captured forward and backward with parts, as the eager calls."""
    d, T, V = (1032, 136, 3336, 1288), 150, 1500
    H, W, y, dl = inputs(d, T, V, seed=3)
    op = mls.HeadLogp(d, T, V)

    def call():
        op.forward(H, W, y)
        op.backward(H, W, y, dl)

    call()
    want = [t.clone() for t in [op.logp, op.lse, op.peak] + op.dH + op.dW]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call()
    for _ in range(3):
        for t in [op.logp, op.lse] + op.dH + op.dW:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = [op.logp, op.lse, op.peak] + op.dH + op.dW
        assert all(torch.equal(a.view(torch.int32) if a.dtype == torch.float32 else a,
                               b.view(torch.int32) if b.dtype == torch.float32 else b) for a, b in zip(got, want))
    assert mls.mls_get_status() == 0


@pytest.mark.gpu
def test_a_stalled_stage_is_reported_and_the_context_survives():
    """A wait that runs out between the parts of a reduction ends the kernel with its status."""
    lines = [line.split() for line in _child(STALL.replace("64", "1352")).splitlines()]
    stalled = [line for line in lines if line[:1] == ["STALLED"]]
    assert [line[1] for line in stalled] == ["fwd", "bwd"]
    assert all(int(line[2]) & B.MLS_STATUS_TIMEOUT for line in stalled)
    assert ["CLEAN", "0", "True"] in lines
