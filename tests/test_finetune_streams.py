"""Calls that the documentation allows on several streams at once, with an object each, and
as the first calls of a process inside a stream capture; and a log-probability call whose
pipeline wait runs out, reported without harm to the context (see test_timeout.py)."""
import os
import subprocess
import sys

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _calls(seed):
    """One call of each operator on its own inputs: (call, outputs)."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def r(*s):
        return torch.randn(*s, generator=g, device="cuda")

    T, V, d, n = 1200, 1500, (64, 136), 9
    x, w, dy = r(T, 136).bfloat16(), r(136).bfloat16(), r(T, 136).bfloat16()
    norm = mls.LayerNorm(T, 136)
    H, W = [r(T, k).bfloat16() for k in d], [(0.2 * r(V, k)).bfloat16() for k in d]
    y = torch.randint(-1, V, (T,), generator=g, device="cuda", dtype=torch.int32)
    dl = r(2, T)
    logp = mls.HeadLogp(d, T, V)
    old, adv = r(2, T), r(n)
    start = torch.randint(0, T + 1, (n + 1,), generator=g, device="cuda").sort().values.to(torch.int32)
    pol = mls.PolicyLoss(T, V, M=2, B=n, agg="seq", adv_per_seq=True)
    raw = [r(30000), r(501).bfloat16()]
    grads = [t.clone() for t in raw]
    clip = mls.GradClip(grads)

    def call():
        norm.forward(x, w, w)
        norm.backward(x, dy, w)
        logp.forward(H, W, y)
        logp.backward(H, W, y, dl)
        pol(old, old + 0.1, adv, y, seq_start=start)
        for a, b in zip(grads, raw):
            a.copy_(b)
        clip(2.0)

    outs = [norm.y, norm.dx, norm.dgain, norm.dbias, logp.logp, logp.lse, *logp.dH, *logp.dW, pol.loss,
            pol.tok_loss, pol.diag, pol.dlogp, clip.stats, *grads]
    return call, outs


def test_two_streams_at_once():
    a, b = _calls(1), _calls(2)
    want = []
    for call, outs in (a, b):
        call()
        torch.cuda.synchronize()
        want.append([t.clone() for t in outs])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for t in a[1] + b[1]:
        t.fill_(0.5)
    torch.cuda.synchronize()
    for _ in range(10):
        for s, (call, _) in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                call()
    torch.cuda.synchronize()
    for (_, outs), w in zip((a, b), want):
        assert all(torch.equal(x, y) for x, y in zip(outs, w))
    assert mls.mls_get_status() == 0


def test_another_current_device_is_refused(monkeypatch):
    """An object's calls run on the device that it was made on, or not at all."""
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    norm, clip = mls.LayerNorm(4, 64, gain=False, bias=False), mls.GradClip([x])
    index = torch.cuda.current_device()
    monkeypatch.setattr(B, "_get_device", lambda: index + 1)
    for call in (lambda: norm.forward(x), lambda: norm.backward(x, x), lambda: clip(1.0),
                 lambda: mls.mls_layer_norm_fwd(x, None, None, 1e-5, x)):
        with pytest.raises(ValueError, match="current device"):
            call()


CAPTURE = r"""
import sys
sys.path.insert(0, {root!r}); sys.path.insert(0, {root!r} + "/tests")
import torch
from test_finetune_streams import _calls
call, outs = _calls(3)
s = torch.cuda.Stream()
s.wait_stream(torch.cuda.current_stream())
with torch.cuda.stream(s):
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call()
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in outs]
call()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, outs))
print("CAPTURED")
"""

STALL = r"""
import os, sys
sys.path.insert(0, {root!r})
import torch
import paper_2608_09703_gb300 as mls
H = [torch.randn(300, 64, device="cuda").bfloat16()]
W = [torch.randn(1000, 64, device="cuda").bfloat16()]
y = torch.zeros(300, dtype=torch.int32, device="cuda")
dl = torch.ones(1, 300, device="cuda")
op = mls.HeadLogp((64,), 300, 1000)
want = [t.clone() for t in (op.forward(H, W, y), *op.backward(H, W, y, dl)[0], *op.dW)]
torch.cuda.synchronize()
for which in ("fwd", "bwd"):
    os.environ["MLS_TEST_STALL_FIRST_STAGE"] = "1"
    op.forward(H, W, y) if which == "fwd" else op.backward(H, W, y, dl)
    torch.cuda.synchronize()
    print("STALLED", which, mls.mls_get_status())
    del os.environ["MLS_TEST_STALL_FIRST_STAGE"]
got = [op.forward(H, W, y), *op.backward(H, W, y, dl)[0], *op.dW]
torch.cuda.synchronize()
print("CLEAN", mls.mls_get_status(), all(torch.equal(a, b) for a, b in zip(got, want)))
"""


def _child(code):
    env = dict(os.environ)
    env.pop("MLS_TEST_STALL_FIRST_STAGE", None)
    r = subprocess.run([sys.executable, "-c", code.format(root=ROOT)], env=env, capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    return r.stdout


def test_first_calls_of_a_process_inside_a_capture():
    assert "CAPTURED" in _child(CAPTURE)


def test_a_stalled_stage_is_reported_and_the_context_survives():
    lines = [l.split() for l in _child(STALL).splitlines()]
    stalled = [l for l in lines if l[:1] == ["STALLED"]]
    assert [l[1] for l in stalled] == ["fwd", "bwd"]
    assert all(int(l[2]) & B.MLS_STATUS_TIMEOUT for l in stalled)
    assert ["CLEAN", "0", "True"] in lines
