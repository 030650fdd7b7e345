"""Sizes past 32 bits are refused, not cut.  CPU only."""
import pytest
import torch

import paper_2407_16847_amd as splat


@pytest.mark.parametrize("kw", [dict(max_len=2 ** 32 + 16), dict(rot_dim=2 ** 32 + 64),
                                dict(ramp=(1.0, 4.0), original_len=2 ** 32 + 8), dict(max_len=-2 ** 32 + 8)])
def test_rotary(kw):
    with pytest.raises((ValueError, splat.SplatError)):
        splat.Rotary(**{**dict(max_len=64, rot_dim=64), **kw})


@pytest.mark.parametrize("at", range(4))
def test_workspace(at):
    a = splat.Acsr(splat.Pattern.window(64, 4), grad=True)
    args = [1, 4, 2, 64]
    splat.decode_workspace(a, *args)
    args[at] += 2 ** 32
    with pytest.raises((ValueError, splat.SplatError)):
        splat.decode_workspace(a, *args)


@pytest.mark.parametrize("at", range(3))
def test_shared_groups(at):
    a = splat.Acsr(splat.Pattern.window(64, 4), grad=True)
    args = [1, 4, 64]
    splat.bwd_shared(a, torch.bfloat16, *args)
    args[at] += 2 ** 32
    with pytest.raises((ValueError, splat.SplatError)):
        splat.bwd_shared(a, torch.bfloat16, *args)
