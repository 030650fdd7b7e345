"""The transposed plan at large strides, and that the GPU cases of
test_gpu_grad_rows.py reach what they are for.  CPU only."""
import time

import numpy as np
import pytest
import torch

import paper_2407_16847_amd as splat
import test_gpu_grad as gpu
import test_gpu_grad_rows as rows
import test_host_grad_plan as plan
from oracle import masks as om

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


def far_pair(L, gap):
    """The diagonal, and one row with a second key `gap` further on."""
    return splat.Pattern.from_terms(L, [dict(lo_i=1, hi_i=1), dict(row_lo=0, row_hi=1, hi_c=gap, stride=gap)])


@pytest.mark.parametrize("pattern,L", [
    (far_pair(65536, 30000), 65536), (splat.Pattern.dilated(65536, 1, 30000), 65536),
    (splat.Pattern.dilated(65536, 1, 8000), 65536), (splat.Pattern.window(65536, 16), 65536),
    (splat.Pattern.dilated(4096, 256, 2), 4096), (splat.Pattern.dilated(1024, 32, 64), 1024)])
def test_key_groups_stay_filled(pattern, L):
    """Large strides do not cut the keys into groups of two or three, and the
    transposed plan takes host time like the plan itself (0.1 s here at the most;
    a pass over all rows for each group takes 5 to 18 s where the groups are many)."""
    t = [time.process_time()]
    splat.Acsr(pattern)
    t.append(time.process_time())
    a = splat.Acsr(pattern, grad=True)
    t.append(time.process_time())
    g, _, tiles, _, _ = a.export_grad_plan()
    assert len(g) <= 2 * max(L // 128, 32)
    assert len(tiles) <= 4 * a.nnz // 64 + 2 * len(g)
    assert t[2] - t[1] <= 2 * (t[1] - t[0]) + 1.0


@pytest.mark.parametrize("kind,params,L", [
    ("dilated", {"w": 3, "dilation": 100}, 300), ("dilated", {"w": 1, "dilation": 299}, 300),
    ("dilated", {"w": 2, "dilation": 130}, 700), ("dilated", {"w": 40, "dilation": 16}, 640),
    ("strided_local", {"local": 7, "stride": 200}, 900)])
def test_strides_past_a_group(kind, params, L):
    a = splat.Acsr(splat.Pattern.named(kind, params, L), grad=True)
    assert np.array_equal(plan._dense(a), om.dense_mask(kind, params, L).astype(np.int64))


def test_one_far_pair():
    a = splat.Acsr(far_pair(500, 333), grad=True)
    M = np.eye(500, dtype=np.int64)
    M[0, 333] = 1
    assert np.array_equal(plan._dense(a), M)


@pytest.mark.parametrize("BH", [1, 200, 5000, 65535])
def test_long_groups_keep_launches_within_their_limit(BH):
    """Groups that take four workgroups do not push a launch past 2^24 of them."""
    for L, w in ((4096, 512), (65536, 40)):
        a = splat.Acsr(splat.Pattern.window_global(L, w, 64), grad=True)
        n = (len(a.export_plan()[0]), len(a.export_grad_plan()[0]))
        for take, all_ in zip(splat.bwd_shared(a, BF16, 1, BH, 64), n):
            assert take == 0 or (all_ + 3 * take) * BH < 2 ** 24
