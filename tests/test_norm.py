"""Layer norm, forward and backward, against the definition in 64 bits.

Tolerances, element by element, from the arithmetic: with u = 2^-24 and ut half a
step of the storage type, a row sum of d values in per-lane chains has a relative
error of at most K u, K = d / 32 + 16 (a chain and the butterfly), so
  |mu - mu'| <= K u mean|x|,  |r - r'| <= K u r,  |xh - xh'| <= K u (|xh| + S)
with S = 1 + r mean|x|; y adds its own rounding ut |y|.  The column sums over T rows
have at most T u of the sum of their terms' sizes.
"""
import ctypes

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from paper_2608_09703_gb300 import build as mbuild

U = 2.0 ** -24


def reference(x, gain, bias, dy, eps):
    """y, mean, rstd, dx, dgain, dbias and the tolerance of each, in 64 bits."""
    ut, d, T = torch.finfo(x.dtype).eps / 2, x.shape[1], x.shape[0]
    x, dy = x.double(), dy.double()
    g = torch.ones(d, dtype=torch.float64, device=x.device) if gain is None else gain.double()
    b = torch.zeros(d, dtype=torch.float64, device=x.device) if bias is None else bias.double()
    mu = x.mean(1, keepdim=True)
    r = 1 / ((x - mu).square().mean(1, keepdim=True) + eps).sqrt()
    xh = (x - mu) * r
    y = xh * g + b
    h = dy * g
    a1, a2 = h.mean(1, keepdim=True), (h * xh).mean(1, keepdim=True)
    dx = r * (h - a1 - xh * a2)
    K = (d / 32 + 16) * U * 1.01
    ax = x.abs().mean(1, keepdim=True)
    S = 1 + r * ax
    w = xh.abs() + S
    tol = dict(
        y=ut * y.abs() + K * (g.abs() * w + y.abs() + b.abs()),
        mean=K * ax[:, 0] + 1e-45, rstd=K * (r * (1 + (K * ax * r) ** 2))[:, 0],
        dx=ut * dx.abs() + 2 * K * r * (h.abs() + h.abs().mean(1, keepdim=True)
                                        + w * (h.abs() * w).mean(1, keepdim=True)),
        dgain=((T + 8) * U + K) * (dy.abs() * w).sum(0) + 1e-45,
        dbias=(T + 8) * U * dy.abs().sum(0) + 1e-45)
    return dict(y=y, mean=mu[:, 0], rstd=r[:, 0], dx=dx, dgain=(dy * xh).sum(0), dbias=dy.sum(0)), tol


def inputs(T, d, dtype, gain, bias, seed=0, mean=0.3, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x = (r(T, d) * scale + mean * scale).to(dtype)
    return (x, (1 + 0.2 * r(d)).to(dtype) if gain else None, (0.3 * r(d)).to(dtype) if bias else None,
            r(T, d).to(dtype))


def close(name, got, want, tol):
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), f"{name}: {int(bad.sum())} values off, worst {float((err / tol).max()):.3g} times the bound"


def check(x, gain, bias, dy, eps=1e-5, op=None):
    T, d = x.shape
    op = op or mls.LayerNorm(T, d, eps=eps, gain=gain is not None, bias=bias is not None, dtype=x.dtype)
    for t in (op.y, op.mean, op.rstd, op.dx, op.dgain, op.dbias):
        if t is not None:
            t.fill_(float("nan"))
    op.forward(x, gain, bias)
    op.backward(x, dy, gain)
    want, tol = reference(x, gain, bias, dy, eps)
    for k in want:
        got = getattr(op, k)
        if got is not None:
            close(k, got, want[k], tol[k])
    return op


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,d", [(1, 8), (1, 16384), (2, 64), (1, 32), (5, 72), (67, 56), (130, 128), (1001, 104), (3001, 40), (3, 520), (5, 4104), (7, 1024), (33, 256),
                                 (130, 2056), (257, 1000), (300, 8192), (1531, 328), (2500, 64), (70, 16392),
                                 (1, 8200), (153, 8200), (400, 12296), (76, 16384), (77, 16000),
                                 (9, 40000)])
def test_against_the_definition(T, d, dtype):
    check(*inputs(T, d, dtype, True, True, seed=T + d))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [384, 392, 640, 648, 768, 776, 1280, 1288, 1536, 1544, 2560, 2568, 4096, 5120, 5128, 6144, 6152, 10240, 10248,
                               12288, 16400, 24576, 24584, 32768, 32776])
def test_either_side_of_each_split(d, dtype):
    """The last width of each number of warps and vectors a lane, and the first of the next."""
    check(*inputs(11, d, dtype, True, True, seed=d))


@pytest.mark.gpu
@pytest.mark.parametrize("gain,bias", [(False, False), (True, False), (False, True)])
def test_optional_parameters(gain, bias):
    x, g, b, dy = inputs(77, 392, torch.bfloat16, gain, bias)
    op = check(x, g, b, dy)
    assert (op.dgain is None) == (not gain) and (op.dbias is None) == (not bias)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_far_mean_constant_rows_and_scales(dtype):
    # a mean a thousand times the spread: one pass over x and x^2 would lose everything
    check(*inputs(40, 776, dtype, True, True, mean=1000.0))
    check(*inputs(40, 776, dtype, True, True, scale=1e-6), eps=1e-12)
    check(*inputs(40, 776, dtype, True, True, scale=1e6))
    x, g, b, dy = inputs(4, 264, dtype, True, True)
    x[1] = 0.0
    x[2] = 3.0
    op = mls.LayerNorm(4, 264, dtype=dtype)
    y = op.forward(x, g, b)
    assert torch.equal(y[1], b) and torch.equal(y[2], b)  # no spread: the bias is left
    want, tol = reference(x[:2], g, b, dy[:2], 1e-5)
    close("y", y[:2], want["y"], tol["y"])


@pytest.mark.gpu
def test_rows_with_infinities_or_nan_stay_alone():
    x, g, b, dy = inputs(9, 520, torch.bfloat16, True, True)
    x[3, 17], x[6, 0] = float("inf"), float("nan")
    op = mls.LayerNorm(9, 520)
    y = op.forward(x, g, b)
    assert torch.isnan(y[3]).all() and torch.isnan(y[6]).all()
    keep = [0, 1, 2, 4, 5, 7, 8]
    want, tol = reference(x[keep], g, b, dy[keep], 1e-5)
    close("y", y[keep], want["y"], tol["y"])
    dx, _, _ = op.backward(x, dy, g)
    close("dx", dx[keep], want["dx"], tol["dx"])


@pytest.mark.gpu
@pytest.mark.parametrize("T,d", [(50, 264), (50, 9000), (600, 2048), (40, 16640)])
def test_in_place(T, d):
    """y may be x and dx may be dy."""
    x, g, b, dy = inputs(T, d, torch.bfloat16, True, True)
    op = check(x, g, b, dy)
    x2, dy2 = x.clone(), dy.clone()
    mls.mls_layer_norm_fwd(x2, g, b, op.eps, x2)
    assert torch.equal(x2, op.y)
    dg, db = torch.empty_like(op.dgain), torch.empty_like(op.dbias)
    mls.mls_layer_norm_bwd(x, g, dy2, op.mean, op.rstd, dy2, dg, db, op.ws)
    assert torch.equal(dy2, op.dx) and torch.equal(dg, op.dgain) and torch.equal(db, op.dbias)


@pytest.mark.gpu
def test_gradient_against_differences():
    """Central differences of the definition in 64 bits, along random directions."""
    x, g, b, dy = inputs(3, 72, torch.float32, True, True, seed=5)
    op = check(x, g, b, dy)
    gen = torch.Generator(device="cuda").manual_seed(6)

    def value(x, g, b):
        mu = x.mean(1, keepdim=True)
        xh = (x - mu) / ((x - mu).square().mean(1, keepdim=True) + op.eps).sqrt()
        return float(((xh * g + b) * dy.double()).sum())

    args = [x.double(), g.double(), b.double()]
    for i, grad in enumerate((op.dx, op.dgain, op.dbias)):
        v = torch.randn(args[i].shape, generator=gen, device="cuda", dtype=torch.float64)
        up, down = list(args), list(args)
        h = 1e-5
        up[i], down[i] = args[i] + h * v, args[i] - h * v
        want = (value(*up) - value(*down)) / (2 * h)
        got = float((grad.double() * v).sum())
        # fp32 gradients (1e-6 of their size), h^2 of the difference, 2^-52 / h of its rounding
        assert abs(got - want) <= 2e-6 * float((grad.double() * v).abs().sum()) + 1e-7


@pytest.mark.gpu
def test_no_rows():
    op = mls.LayerNorm(0, 64)
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    op.forward(x, w, w)
    op.dgain.fill_(5.0), op.dbias.fill_(5.0)
    op.backward(x, x, w)
    assert not op.dgain.any() and not op.dbias.any()


@pytest.mark.gpu
def test_repeatable_streams_and_graph():
    x, g, b, dy = inputs(700, 1032, torch.bfloat16, True, True)
    op = check(x, g, b, dy)
    want = [t.clone() for t in (op.y, op.dx, op.dgain, op.dbias)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            op.forward(x, g, b)
            op.backward(x, dy, g)
    for _ in range(3):
        for t in (op.y, op.dx, op.dgain, op.dbias):
            t.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip((op.y, op.dx, op.dgain, op.dbias), want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = torch.empty_like(x)
    mls.mls_layer_norm_fwd(x, g, b, op.eps, y, stream=side)
    side.synchronize()
    assert torch.equal(y, want[0])


# ------------------------------------------------------------------ refusals (CPU)
def test_refusals_of_the_library():
    mbuild.build()
    L = B.lib()
    p, q, m = 0x1000, 0x2000, 0x3000

    def fwd(T=4, d=64, dt=0, eps=1e-5, x=p, gain=p, bias=p, y=q, mean=m, rstd=m):
        return L.mls_layer_norm_fwd(T, d, dt, eps, x, gain, bias, y, mean, rstd, None)

    for kw in (dict(T=-1), dict(T=1 << 31), dict(d=0), dict(dt=2), dict(eps=-1.0), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None)):
        assert fwd(**kw) == B.MLS_ERR_ARG, kw
    assert fwd(d=60) == B.MLS_ERR_UNSUPPORTED and fwd(d=6, dt=1) == B.MLS_ERR_UNSUPPORTED
    assert fwd(d=(1 << 28) + 8) == B.MLS_ERR_UNSUPPORTED and fwd(d=(1 << 31) - 8) == B.MLS_ERR_UNSUPPORTED
    assert B.mls_layer_norm_workspace_size(1, (1 << 28) + 8) == 0
    for kw in (dict(x=p + 8), dict(gain=p + 8), dict(bias=p + 2), dict(y=q + 4), dict(mean=m + 2)):
        assert fwd(**kw) == B.MLS_ERR_ALIGN, kw

    def bwd(T=4, d=64, dt=0, x=p, gain=p, dy=p, mean=m, rstd=m, dx=q, dgain=q, dbias=q):
        return L.mls_layer_norm_bwd(T, d, dt, x, gain, dy, mean, rstd, dx, dgain, dbias, 0x10000, 1 << 30, None)

    for kw in (dict(T=-1), dict(d=0), dict(dt=3), dict(x=None), dict(dy=None), dict(dx=None), dict(mean=None),
               dict(rstd=None)):
        assert bwd(**kw) == B.MLS_ERR_ARG, kw
    assert bwd(d=60) == B.MLS_ERR_UNSUPPORTED
    for kw in (dict(dy=p + 8), dict(dx=q + 8), dict(dgain=q + 2), dict(rstd=m + 1)):
        assert bwd(**kw) == B.MLS_ERR_ALIGN, kw
    assert B.mls_layer_norm_workspace_size(-1, 64) == 0 and B.mls_layer_norm_workspace_size(10, 0) == 0
    assert B.mls_layer_norm_workspace_size(1 << 20, 64) > 0


@pytest.mark.gpu
def test_refusals_of_the_binding():
    x, g, b, dy = inputs(10, 64, torch.bfloat16, True, True)
    y = torch.empty_like(x)
    with pytest.raises(TypeError):
        mls.mls_layer_norm_fwd(x.half(), g, b, 1e-5, y)
    with pytest.raises(TypeError):
        mls.mls_layer_norm_fwd(x, g.float(), b, 1e-5, y)
    with pytest.raises(ValueError):
        mls.mls_layer_norm_fwd(x, g[:32], b, 1e-5, y)
    with pytest.raises(ValueError):
        mls.mls_layer_norm_fwd(x, g, b, 1e-5, torch.empty(64, 10, dtype=x.dtype, device="cuda").t())
    with pytest.raises(ValueError):
        mls.mls_layer_norm_fwd(x, g.cpu(), b, 1e-5, y)
    op = mls.LayerNorm(10, 64, bias=False)
    with pytest.raises(ValueError):
        op.forward(x, g, b)
    with pytest.raises(ValueError):
        op.forward(x)
    op.forward(x, g)
    with pytest.raises(mls.MLSError) as e:
        mls.mls_layer_norm_bwd(x, g, dy, op.mean, op.rstd, op.dx, op.dgain, None, op.ws[:16])
    assert e.value.code == B.MLS_ERR_WORKSPACE
    with pytest.raises(ValueError):
        mls.LayerNorm(10, 64, backward=False).backward(x, dy, g)


def test_cpu_tensors_are_refused():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        mls.mls_layer_norm_fwd(x, None, None, 1e-5, torch.empty_like(x))
