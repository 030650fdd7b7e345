"""What cache_evict refuses without a GPU.  CPU only: every call here returns before
anything would be launched."""
import ctypes

import pytest
import torch

import paper_2407_16847_amd as splat


def call(dtype=0, B=2, d=64, weights=3 << 20, lengths=4 << 20, budget=16, first=0, recent=0, to=5 << 20, max_to=2,
         kept=6 << 20, left=7 << 20, k=1 << 20, v=2 << 20, table=8 << 20, n_pages=8, heads=2, page=8, max_pages=5):
    cache = (ctypes.c_int64 * 7)(k or 0, v or 0, table or 0, n_pages, heads, page, max_pages)
    return splat.load().splat_cache_evict(dtype, B, d, cache, weights, lengths, budget, first, recent, to, max_to,
                                          kept, left, None)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(B=0), dict(B=32768), dict(weights=None), dict(weights=(3 << 20) + 2),
    dict(lengths=None), dict(budget=0), dict(budget=65537), dict(first=-1), dict(recent=-1), dict(first=9, recent=8),
    dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), dict(max_to=0), dict(max_to=1), dict(budget=17), dict(kept=None),
    dict(left=None), dict(kept=2), dict(k=None), dict(v=None), dict(table=None), dict(n_pages=0), dict(heads=0),
    dict(page=12), dict(page=1 << 17), dict(max_pages=0), dict(k=(1 << 20) + 8),
    # outputs over what the call reads or another output
    dict(v=1 << 20), dict(weights=1 << 20), dict(kept=4 << 20), dict(left=4 << 20), dict(left=6 << 20),
    dict(to=6 << 20), dict(table=3 << 20), dict(left=5 << 20), dict(kept=(2 << 20) + 16)])
def test_refusals(bad):
    assert call(**bad) == 1
    assert splat.load().splat_last_error()


def test_unsupported():
    assert call(d=96) == 2
    assert call(n_pages=1 << 30, heads=2, page=8) == 2      # rows past 32 bits


def test_host_tensors():
    x = torch.zeros(2, 2, 8, 64)
    n = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        splat.cache_evict(x, x, torch.zeros(2, 2, 8), torch.zeros(2, 1, dtype=torch.int32), n, 4)
