"""Failure detection in tree attention without a GPU fault: with the test hook MLS_TEST_STALL_FIRST_STAGE set, each CTA
brings nothing for its first stage of keys.  The wait for it runs out (about 2 s), the CTA's other roles leave, what was
asked for meanwhile lands before its shared memory goes away, and the call reports MLS_STATUS_TIMEOUT, without
MLS_STATUS_DRAIN.  The same process then computes the same bits as before.  A child process, so that the hook
cannot leak into other tests."""
import os
import subprocess
import sys

import pytest

from paper_2608_09703_gb300 import binding as B

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import os, sys
sys.path.insert(0, {root!r})
import torch
import paper_2608_09703_gb300 as mls

def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")

# Widths of one and two pieces, rows of one and two tiles, single tokens; more tiles than stages, and fewer.
for name, dtype, dim, n, heads, length in (
        ("bf16_128", torch.bfloat16, 128, 40, 8, 3000), ("bf16_128_one", torch.bfloat16, 128, 1, 4, 100),
        ("bf16_72", torch.bfloat16, 72, 5, 4, 3000), ("bf16_64", torch.bfloat16, 64, 40, 8, 300),
        ("fp32_16", torch.float32, 128, 9, 8, 3000), ("fp32_16_narrow", torch.float32, 64, 9, 8, 3000),
        ("fp32_4", torch.float32, 128, 1, 8, 3000), ("fp32_4_short", torch.float32, 64, 1, 8, 40)):
    torch.manual_seed(1)
    kv, S = 2, 3
    c = mls.PagedCache(1, S * ((length + n) // 16 + 1), 16, kv, dim, S, (length + n) // 16 + 1, dtype=dtype)
    c.reserve(i32([length + n] * S))
    c.k.normal_()
    c.v.normal_()
    c.compact(i32([length] * S))
    c.reserve(i32([n] * S))
    q = torch.randn(S * n, heads, dim, device="cuda").to(dtype)
    start = i32([n * i for i in range(S + 1)])
    parents = i32([-1] + list(range(n - 1))).repeat(S)
    op = mls.TreeAttention(c, S, S * n, heads)
    want = [t.clone() for t in op(q, start, parents)]
    torch.cuda.synchronize()
    assert mls.mls_get_status() == 0
    os.environ["MLS_TEST_STALL_FIRST_STAGE"] = "1"
    op(q, start, parents)
    torch.cuda.synchronize()
    stalled = mls.mls_get_status()
    del os.environ["MLS_TEST_STALL_FIRST_STAGE"]
    op.out.zero_()
    got = op(q, start, parents)
    torch.cuda.synchronize()
    print("CASE", name, stalled, mls.mls_get_status(), all(torch.equal(a, b) for a, b in zip(got, want)))
"""


def test_stalled_stages_are_reported_and_the_context_survives():
    env = dict(os.environ)
    env.pop("MLS_TEST_STALL_FIRST_STAGE", None)
    r = subprocess.run([sys.executable, "-c", CHILD.format(root=ROOT)], env=env, capture_output=True, text=True,
                       timeout=240)
    assert r.returncode == 0, r.stdout + r.stderr
    cases = [l.split()[1:] for l in r.stdout.splitlines() if l.startswith("CASE")]
    assert len(cases) == 8
    for name, stalled, clean, same in cases:
        assert int(stalled) == B.MLS_STATUS_TIMEOUT, (name, stalled)
        assert int(clean) == 0 and same == "True", name
