"""The norm and the factor of clipping are rounded once: gradients whose squares' sum is exact (equal
powers of two) give the nearest fp32 values of the root and of the quotient."""
import math

import pytest
import torch

import paper_2608_09703_gb300 as mls


@pytest.mark.gpu
@pytest.mark.parametrize("power", [0, -10, 20, -70, 50])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_nearest_values(power, dtype):
    arena = torch.empty(700001, device="cuda", dtype=dtype)
    want, got = [], []
    for i in range(60):
        n = 1 + i * i * 191 + 17 * i
        g = arena[:n].fill_(2.0 ** power)
        norm = math.sqrt(n) * 2.0 ** power
        most = float(torch.tensor((0.1 + 0.013 * i) * norm))
        want.append((norm, min(1.0, most / (norm + 1e-6))))
        got.append(mls.GradClip([g])(most).clone())
    want, got = torch.tensor(want, dtype=torch.float64).float(), torch.stack(got).cpu()
    assert torch.equal(got[:, 0], want[:, 0]), int((got[:, 0] != want[:, 0]).sum())
    assert torch.equal(got[:, 1], want[:, 1]), int((got[:, 1] != want[:, 1]).sum())


@pytest.mark.gpu
def test_ends_of_the_range():
    def clip(value, n, most):
        return mls.GradClip([torch.full((n,), value, device="cuda")])(most).tolist()

    near = lambda v: float(torch.tensor(v, dtype=torch.float64).float())  # noqa: E731
    # a norm past the largest fp32 value, and one a factor of 2^149 from its bound
    big = 1.5 * 2.0 ** 127
    assert clip(big, 5, 2.0 ** 100) == [math.inf, near(2.0 ** 100 / (math.sqrt(5) * big))]
    assert clip(2.0 ** -149, 3, 1.0) == [near(math.sqrt(3) * 2.0 ** -149), 1.0]
    # 1e-6 decides
    norm = math.sqrt(3) * 2.0 ** -20
    assert clip(2.0 ** -20, 3, 2.0 ** -21) == [near(norm), near(2.0 ** -21 / (norm + 1e-6))]
    assert clip(2.0 ** -60, 7, 2.0 ** -22) == [near(math.sqrt(7) * 2.0 ** -60), near(2.0 ** -22 / (math.sqrt(7) * 2.0 ** -60 + 1e-6))]
    # bounds that need nothing, however large or near
    assert clip(1.0, 4, 3e38) == [2.0, 1.0] and clip(1.0, 4, 2.0000011) == [2.0, 1.0]
    assert clip(0.0, 4, 1e-7) == [0.0, near(float(torch.tensor(1e-7)) / 1e-6)]
