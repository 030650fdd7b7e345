"""How cache_weights goes about a launch.  CPU only."""
import pytest
import torch

import paper_2407_16847_amd as splat

BF16, F32 = torch.bfloat16, torch.float32


def causal(L):
    return splat.Acsr(splat.Pattern.from_terms(L, [dict(hi_i=1)]))


@pytest.mark.parametrize("dtype,d,held", [(BF16, 64, 1024), (BF16, 128, 512), (F32, 64, 512), (F32, 128, 256)])
def test_parts_fit_the_chip(dtype, d, held):
    """As many workgroups as are there at a time, by their LDS, and none in a second turn;
    where there is little to do, one for four units at least."""
    a = causal(4096)
    for heads in (1, 3, 7, 8, 20, 24, 32, 48, 100, 255, 257, 600, 1025):
        route, parts = splat.weights_route(a, dtype, 1, heads, heads, 1, d, 4096)
        assert route == "units" and 1 <= parts <= 32
        assert parts == 1 or heads * parts <= held
        assert parts == 32 or heads * (parts + 1) > held
        assert splat.weights_route(a, dtype, 1, heads, heads, 1, d, 100)[1] == 1
    assert splat.weights_route(a, dtype, 32, 32, 8, 1, d, 4096)[1] == held // 8


def test_refusals():
    a = causal(100)
    for args in ((0, 4, 4, 1, 64, 100), (1, 4, 3, 1, 64, 100), (1, 4, 4, 0, 64, 100), (1, 4, 4, 1, 96, 100), (1, 4, 4, 1, 64, 0)):
        with pytest.raises(splat.SplatError):
            splat.weights_route(a, BF16, *args)
    assert splat.load().splat_debug_weights(a.handle, 1, 1, 4, 4, 1, 64, 100, None) == 1
