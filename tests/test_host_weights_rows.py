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


def test_faster_side():
    """Measured launches on both sides of the choice, over tables of the masks' length."""
    window = lambda L, w: splat.Acsr(splat.Pattern.from_terms(L, [dict(lo_i=1, lo_c=-w, hi_i=1)]))
    for a, B, heads, d, units, tiles in (
            (causal(4096), 1, 4, 64, 160, 256), (causal(4096), 1, 16, 64, 384, 512), (causal(4096), 1, 32, 64, 320, 448),
            (causal(4096), 8, 16, 64, 384, 512), (causal(1024), 1, 32, 64, 160, 256), (window(4096, 256), 1, 16, 64, 192, 256),
            (window(4096, 1500), 1, 24, 64, 192, 256), (causal(4096), 1, 4, 128, 96, 192), (causal(4096), 1, 16, 128, 320, 384),
            (causal(4096), 8, 16, 128, 256, 448), (window(4096, 256), 1, 24, 128, 160, 192), (causal(1024), 1, 12, 128, 96, 160)):
        room = a._info["L"]
        assert splat.weights_route(a, BF16, B, heads, heads, units, d, room)[0] == "units", (B, heads, d, units)
        assert splat.weights_route(a, BF16, B, heads, heads, tiles, d, room)[0] == "tiles", (B, heads, d, tiles)
        assert splat.weights_route(a, F32, B, heads, heads, tiles, d, room)[0] == "units"
