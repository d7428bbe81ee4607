"""A clipping object follows its tensors when they are given other memory, at the same address
and of the same count too: of another type, or strided.  The memory is one arena, so that no
call, whatever it takes the tensor for, leaves it."""
import math

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B

U = 2.0 ** -24


def test_places_tell_type_and_strides():
    b = torch.zeros(64)
    g = b[:10]
    before = B._places([g])
    g.data = b[::2][:10]
    assert g.data_ptr() == b.data_ptr() and g.numel() == 10
    assert B._places([g]) != before
    g.data = b[:10]
    assert B._places([g]) == before
    g.data = b.view(torch.bfloat16)[:10]
    assert g.data_ptr() == b.data_ptr() and g.numel() == 10
    assert B._places([g]) != before
    m = torch.zeros(4, 8)
    n = m[:]
    before = B._places([n])
    n.data = m.view(8, 4).t()  # dense, in another order
    assert B._places([n]) != before


@pytest.mark.gpu
def test_same_address_other_type():
    arena = torch.full((4096,), 2.0, device="cuda")
    g = arena[:1000]
    op = mls.GradClip([g])
    op(1e9)
    halves = arena.view(torch.bfloat16)
    halves.fill_(3.0)
    g.data = halves[:1000]
    norm, coef = op(1.0).tolist()
    want = math.sqrt(1000 * 9.0)
    assert abs(norm - want) <= 8 * U * want and abs(coef - 1 / (want + 1e-6)) <= 10 * U * coef
    assert bool((halves[1000:] == 3.0).all())  # behind the tensor
    assert torch.equal(g, torch.full_like(g, 3.0 * coef))
    g.data = arena.view(torch.int32)[:1000]
    with pytest.raises(TypeError):
        op(1.0)


@pytest.mark.gpu
def test_same_address_strided():
    arena = torch.full((4096,), 2.0, device="cuda")
    g = arena[:1000]
    op = mls.GradClip([g])
    op(1e9)
    keep = arena.clone()
    g.data = arena[::2][:1000]
    with pytest.raises(ValueError):
        op(1.0)
    assert torch.equal(arena, keep)
    g.data = arena[:1000]
    norm, _ = op(1.0).tolist()
    assert abs(norm - math.sqrt(4000.0)) <= 8 * U * norm
