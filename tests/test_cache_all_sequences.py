"""free() without a list of sequences, on caches of more sequences than a call with a list may name."""
import ctypes

import pytest
import torch

import paper_2608_09703_gb300 as mls
from paper_2608_09703_gb300 import binding as B
from test_cache import i32


@pytest.fixture(autouse=True)
def clean_status(request):
    """Each test begins with no status of another."""
    if "gpu" in request.keywords:
        mls.mls_get_status()


def test_the_limit_is_that_of_a_list():
    """What the host can see (no GPU): a list of too many entries, or more sequences than there are, is refused."""
    L, P = B.lib(), 0x1000
    c = B.mls_cache(2, 10, 16, 2, 64, B.MLS_BF16, 20000, 4, P, P, P, P, P, P, P)
    most = B.MLS_CACHE_MAX_ENTRIES
    assert L.mls_cache_free(ctypes.byref(c), most + 1, ctypes.c_void_p(P), None) == B.MLS_ERR_UNSUPPORTED
    assert L.mls_cache_free(ctypes.byref(c), 20001, None, None) == B.MLS_ERR_ARG
    assert L.mls_cache_reserve(ctypes.byref(c), most + 1, None, ctypes.c_void_p(P), None) == B.MLS_ERR_UNSUPPORTED
    if not torch.cuda.is_available():  # past the checks, which is where it finds no device
        assert L.mls_cache_free(ctypes.byref(c), 20000, None, None) == B.MLS_ERR_CUDA


@pytest.mark.gpu
@pytest.mark.parametrize("seqs", [B.MLS_CACHE_MAX_ENTRIES, B.MLS_CACHE_MAX_ENTRIES + 1, 20000])
def test_free_all(seqs):
    c = mls.PagedCache(1, seqs + 5, 8, 1, 8, seqs, 2)
    for at in range(0, seqs, B.MLS_CACHE_MAX_ENTRIES):
        ids = torch.arange(at, min(at + B.MLS_CACHE_MAX_ENTRIES, seqs), dtype=torch.int32, device="cuda")
        ones = torch.ones_like(ids)
        c.reserve(ones, ids)
        c.compact(ones, seqs=ids)
    assert int(c.len.sum()) == int(c.held.sum()) == int(c.refs.sum()) == seqs
    c.free()
    assert not c.len.any() and not c.held.any() and not c.refs.any() and bool((c.table == -1).all())
    bits = [b & 0xffffffff for b in c.free_bits.tolist()]
    assert sum(bin(b).count("1") for b in bits) == seqs + 5
    assert mls.mls_get_status() == 0
