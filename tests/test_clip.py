"""Global gradient norm and clipping against the definition in 64 bits.

Tolerances with u = 2^-24: the squares of 32 values are summed in four chains of 8 and
added, 12 u of the sum at most, then in 64 bits; the root halves that and is rounded:
8 u of the norm.  The factor adds its own rounding, 10 u.  A gradient is multiplied in
32 bits and rounded to its type once.
"""
import ctypes
import math

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from paper_2608_09703_gb300 import build as mbuild

U = 2.0 ** -24


def tensors(sizes, seed=0, dtypes=(torch.bfloat16, torch.float32), offset=0, scale=1.0):
    """Views of one buffer per type, packed without padding, `offset` values from its start."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for k, dt in enumerate(dtypes):
        mine = sizes[k::len(dtypes)]
        buf = torch.empty(offset + sum(mine) + 16, dtype=dt, device="cuda").fill_(7.0)
        at = offset
        for n in mine:
            buf[at:at + n] = (torch.randn(n, generator=g, device="cuda") * scale).to(dt)
            out.append(buf[at:at + n])
            at += n
    return out


def check(grads, max_norm):
    before = [g.clone() for g in grads]
    op = mls.GradClip(grads)
    norm, coef = op(max_norm).tolist()
    want = math.sqrt(sum(float(g.double().square().sum()) for g in before))
    if want > torch.finfo(torch.float32).max:  # reported in 32 bits, which end at 3.4e38; c is not affected
        assert norm == math.inf
    else:
        assert abs(norm - want) <= 8 * U * want + 2.0 ** -150  # half a step of the smallest fp32 values
    c = min(1.0, max_norm / (want + 1e-6)) if math.isfinite(max_norm) else 1.0
    assert abs(coef - c) <= 10 * U * c
    for g, b in zip(grads, before):
        if coef == 1.0:
            assert torch.equal(g, b)
            continue
        w = b.double() * c
        fi = torch.finfo(g.dtype)
        tol = (fi.eps / 2 + 12 * U) * w.abs() + fi.tiny * fi.eps
        assert bool(((g.double() - w).abs() <= tol).all())
    return norm, coef


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[1], [7], [8191], [8192], [8193], [16385, 1], [3, 0, 5, 0], [100003, 17, 64, 9000],
                                   [1] * 50, [0, 0]])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_sizes_and_alignments(sizes, offset):
    for max_norm in (1e-2, 1e9, math.inf):
        check(tensors(sizes, seed=len(sizes), offset=offset), max_norm)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1023, 1024, 1025, 2500])
def test_many_tensors(n):
    """More tensors than one launch's table."""
    check(tensors([1 + (i * 37) % 300 for i in range(n)], seed=n), 0.5)


@pytest.mark.gpu
def test_nothing_beside_the_tensors_changes():
    g = tensors([1001, 30, 77, 5], seed=2, offset=5)
    bufs = {t.untyped_storage().data_ptr(): t for t in g}
    mls.GradClip(g)(1e-3)
    for t in bufs.values():
        whole = torch.empty(0, dtype=t.dtype, device="cuda").set_(t.untyped_storage())
        assert bool((whole[:5] == 7).all()) and bool((whole[-16:] == 7).all())


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e-30, 1e-22, 1e-12, 1e15, 1e30, 3e37])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_squares_beyond_fp32(scale, dtype):
    """Norms whose squares overflow or vanish in 32 bits."""
    norm, _ = check(tensors([5000, 300], seed=1, dtypes=(dtype,), scale=scale), scale)
    assert norm > 0 and math.isfinite(norm) == (scale < 3e37)  # 72 x 3e37 is past fp32's largest value


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e-44, 1e-41, 1e-38, 1e-34, 1e-13, 1e-12])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_smallest_gradients(scale, dtype):
    """Down to the smallest values of either type (bf16 has none at 1e-44), and across the
    border at which squares are taken of scaled values."""
    norm, _ = check(tensors([50000, 300, 8192], seed=1, dtypes=(dtype,), scale=scale), math.inf)
    assert (norm > 0) == (dtype is torch.float32 or scale > 1e-43)


@pytest.mark.gpu
def test_large_next_to_small_and_zeros():
    a = torch.zeros(20000, device="cuda")
    a[3] = 1e25
    b = torch.full((30000,), 1e-30, device="cuda")
    check([a, b], 1.0)
    z = torch.zeros(40000, device="cuda", dtype=torch.bfloat16)
    assert check([z], 1.0) == (0.0, 1.0)


@pytest.mark.gpu
def test_nan_and_infinity():
    g = tensors([9000, 50], seed=4)
    g[0][777] = float("nan")
    op = mls.GradClip(g)
    norm, coef = op(1.0).tolist()
    assert math.isnan(norm) and math.isnan(coef) and all(torch.isnan(t).all() for t in g)
    g = tensors([9000, 50], seed=4)
    g[1][7] = -float("inf")
    norm, coef = mls.GradClip(g)(1.0).tolist()
    assert norm == math.inf and coef == 0
    assert math.isnan(g[1][7]) and not g[0].any() and not g[1][:7].any()
    g = tensors([300], seed=4, dtypes=(torch.float32,))
    g[0][0] = float("nan")
    keep = g[0].clone()
    norm, coef = mls.GradClip(g)(math.inf).tolist()  # only the norm: nothing is touched
    assert math.isnan(norm) and coef == 1 and torch.equal(g[0][1:], keep[1:])


@pytest.mark.gpu
def test_repeatable_captured_and_two_at_once():
    sizes = [70001, 13, 4096, 250000]
    g1, g2 = tensors(sizes, seed=1), tensors(sizes, seed=2)
    keep1, keep2 = [t.clone() for t in g1], [t.clone() for t in g2]
    op1, op2 = mls.GradClip(g1), mls.GradClip(g2)
    want = [s.clone() for s in (op1(0.7), op2(0.3))]
    out1, out2 = [t.clone() for t in g1], [t.clone() for t in g2]
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    s1.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s1):
        with torch.cuda.graph(graph, stream=s1):
            op1(0.7)
    for _ in range(5):
        for t, k in zip(g1 + g2, keep1 + keep2):
            t.copy_(k)
        for s in (s1, s2):
            s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s1):
            graph.replay()
        op2(0.3, stream=s2)
        torch.cuda.synchronize()
        assert torch.equal(op1.stats, want[0]) and torch.equal(op2.stats, want[1])
        assert all(torch.equal(a, b) for a, b in zip(g1 + g2, out1 + out2))


# ------------------------------------------------------------------ refusals (CPU)
def test_refusals_of_the_library():
    mbuild.build()
    L = B.lib()

    def call(ptrs=(0x1000, 0x2000), numel=(8, 8), dtype=(0, 1), max_norm=1.0, stats=0x3000, n=None):
        k = len(ptrs)
        return L.mls_grad_clip(k if n is None else n, (ctypes.c_void_p * k)(*ptrs), (ctypes.c_int64 * k)(*numel),
                               (ctypes.c_int32 * k)(*dtype), max_norm, stats, 0x10000, 1 << 30, None)

    for kw in (dict(n=-1), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=math.nan), dict(stats=None),
               dict(numel=(8, -1)), dict(dtype=(0, 2)), dict(ptrs=(0x1000, None)),
               dict(ptrs=(0x1000, 0x1000)),                       # the same tensor twice
               dict(ptrs=(0x1000, 0x1008), numel=(8, 8)),         # overlapping
               dict(ptrs=(0x1020, 0x1000), numel=(8, 9))):        # the second reaches into the first
        assert call(**kw) == B.MLS_ERR_ARG, kw
    assert call(ptrs=(0x1000, 0x2002)) == B.MLS_ERR_ALIGN and call(ptrs=(0x1001, 0x2000)) == B.MLS_ERR_ALIGN
    assert call(n=16385) == B.MLS_ERR_UNSUPPORTED
    assert call(stats=0x3002) == B.MLS_ERR_ALIGN
    assert L.mls_grad_clip(2, None, None, None, 1.0, 0x3000, 0x10000, 1 << 30, None) == B.MLS_ERR_ARG
    assert B.mls_grad_clip_workspace_size(-1) == 0 and B.mls_grad_clip_workspace_size(16385) == 0
    assert B.mls_grad_clip_workspace_size(16384) > B.mls_grad_clip_workspace_size(1) > 0


def test_refusals_of_the_binding():
    with pytest.raises(ValueError):
        mls.GradClip([])
    with pytest.raises(ValueError):
        mls.GradClip([torch.zeros(4)])


@pytest.mark.gpu
def test_refusals_of_the_binding_on_the_gpu():
    with pytest.raises(TypeError):
        mls.GradClip([torch.zeros(4, dtype=torch.float16, device="cuda")])
    with pytest.raises(ValueError):
        mls.GradClip([torch.zeros(4, 4, device="cuda").t()[1:]])
    with pytest.raises(ValueError):
        mls.GradClip([torch.zeros(4, device="cuda"), torch.zeros(4)])
    g = [torch.ones(100, device="cuda")]
    with pytest.raises(mls.MLSError):
        mls.GradClip(g + g)(1.0)
    assert bool((g[0] == 1).all())
    with pytest.raises(mls.MLSError):
        mls.GradClip(g)(0.0)


@pytest.mark.gpu
def test_tensors_given_other_memory():
    """An object's list follows its tensors, not the memory they had when it was made."""
    g = tensors([5000, 70], seed=9)
    op = mls.GradClip(g)
    op(1.0)
    old = g[0].data
    keep = old.clone()
    g[0].data = torch.full((600,), 3.0, dtype=g[0].dtype, device="cuda")
    g[1].data = g[1].data[:9]
    g[1].fill_(2.0)
    norm, coef = op(1.0).tolist()
    want = math.sqrt(600 * 9.0 + 9 * 4.0)
    assert abs(norm - want) <= 8 * U * want and abs(coef - 1 / (want + 1e-6)) <= 10 * U * coef
    assert torch.equal(old, keep)  # the memory left behind
    g[1].data = torch.zeros(4, 4, dtype=g[1].dtype, device="cuda").t()[:2]
    with pytest.raises(ValueError):
        op(1.0)
