"""Pages are copied between caches of one device only: a kernel that ran on one and wrote to the other's memory would fault.
Two caches of made-up devices, no GPU: the refusal comes before the library is called."""
import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B


def cache_on(index):
    c = object.__new__(mls.PagedCache)
    c.c = B.mls_cache()
    c.home = object.__new__(B._Home)
    c.home.index = index
    return c


@pytest.mark.parametrize("now,own,other", [(0, 0, 1), (1, 1, 0), (1, 0, 1), (1, 0, 0)])
def test_copy_to_another_device(monkeypatch, now, own, other):
    monkeypatch.setattr(B, "_get_device", lambda: now)
    called = []
    monkeypatch.setattr(B, "mls_cache_copy", lambda *a: called.append(a))
    pages = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="current device"):
        cache_on(own).copy(pages, pages, to=cache_on(other))
    assert not called


def test_copy_on_one_device(monkeypatch):
    monkeypatch.setattr(B, "_get_device", lambda: 1)
    called = []
    monkeypatch.setattr(B, "mls_cache_copy", lambda *a: called.append(a))
    pages = torch.zeros(1, dtype=torch.int32)
    a, b = cache_on(1), cache_on(1)
    a.copy(pages, pages, to=b)
    a.copy(pages, pages)
    assert [x[:2] for x in called] == [(a.c, b.c), (a.c, a.c)]
