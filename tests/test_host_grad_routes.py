"""Which of the backward pass's ways through a group the GPU tests' cases reach
(host only), and how the choice goes at sizes where it was measured."""
import ctypes

import pytest
import torch

import paper_2407_16847_amd as splat
import test_gpu_grad as gpu

BF16, F32 = torch.bfloat16, torch.float32


def _shared(kind, params, L, heads, d, B=1):
    a, _ = gpu.make(splat, kind, params, L)
    g, _, _ = a.export_plan()
    return splat.bwd_shared(a, BF16, B, heads, d), (len(g), len(a.export_grad_plan()[0]))


@pytest.mark.parametrize("d", [64, 128])
def test_the_gpu_cases_reach_both_ways(d):
    own, four = set(), set()
    for kind, params, L, heads in gpu.CASES + gpu.LARGE:
        s, n = _shared(kind, params, L, heads, d)
        for k in range(2):
            assert 0 <= s[k] <= n[k]
            if s[k] < n[k]:
                own.add(k)
            if s[k]:
                four.add(k)
            if 0 < s[k] < n[k]:
                four.add(2 + k)
    assert own == {0, 1} and four >= {0, 1, 3}


@pytest.mark.parametrize("case,want", [
    (("window_global", {"w": 512, "n_global": 64}, 4096, 64, 64), (0, 0)),
    (("window_global", {"w": 512, "n_global": 64}, 4096, 16, 64), (1, 1)),
    (("strided_local", {"local": 128, "stride": 128}, 2048, 24, 64), (0, 1)),
    (("dilated", {"w": 256, "dilation": 2}, 4096, 16, 128), (0, 0)),
    (("full", {}, 777, 16, 128), (7, 7)),
])
def test_measured_choices(case, want):
    assert _shared(*case)[0] == want


def test_refusals():
    a = splat.Acsr(splat.Pattern.window(64, 4))
    with pytest.raises(splat.SplatError, match="SPLAT_PLAN_GRAD"):
        splat.bwd_shared(a, BF16, 1, 1, 64)
    a = splat.Acsr(splat.Pattern.window(64, 4), grad=True)
    assert splat.bwd_shared(a, F32, 1, 1, 64) == (0, 0)
    lib, n = splat.load(), (ctypes.c_int32 * 2)()
    for args in ((None, 1, 1, 1, 64, n), (a.handle, 2, 1, 1, 64, n), (a.handle, 1, 0, 1, 64, n),
                 (a.handle, 1, 1, 1, 64, None)):
        assert lib.splat_debug_bwd_shared(*args) == 1
    assert lib.splat_debug_bwd_shared(a.handle, 1, 1, 1, 96, n) == 2
