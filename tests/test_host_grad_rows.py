"""That the GPU cases of test_gpu_grad_rows.py reach what they are for.  CPU only."""
import numpy as np
import pytest
import torch

import paper_2407_16847_amd as splat
import test_gpu_grad as gpu
import test_gpu_grad_rows as rows

BF16 = torch.bfloat16


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,params,L,heads", rows.NO_ROWS)
def test_keys_without_rows_fill_a_workgroup(kind, params, L, heads, d):
    """Groups of 128 keys without a tile, each of one workgroup with four
    wavefronts of keys."""
    a, M = gpu.make(splat, kind, params, L)
    g = a.export_grad_plan()[0]
    empty = (g[:, 2] == g[:, 3])
    assert (empty & (g[:, 1] == 128)).any()
    assert splat.bwd_shared(a, BF16, 1, heads, d)[1] <= int(np.argmax(empty))
