"""What the chunk's calls refuse without a GPU.  CPU only."""
import ctypes

import pytest
import torch

import paper_2407_16847_amd as splat


@pytest.fixture(scope="module")
def acsr():
    return splat.Acsr(splat.Pattern.window(4096, 2000))


def test_workspace(acsr):
    assert splat.chunk_workspace(acsr, torch.bfloat16, 1, 4, 4, 1, 64) > 0      # one row over many keys
    assert splat.chunk_workspace(acsr, torch.bfloat16, 64, 16, 16, 8, 64) == 0  # a full chip
    for args in ((0, 4, 4, 1, 64), (1, 4, 3, 1, 64), (1, 4, 0, 1, 64), (1, 4, 8, 1, 64), (1, 4, 4, 0, 64),
                 (1, 4, 4, 1, 96), (1, 70000, 1, 1, 64), (1, 64, 1, (1 << 18) + 1, 64), (1, 4, 4, -1, 64)):
        with pytest.raises(splat.SplatError):
            splat.chunk_workspace(acsr, torch.float32, *args)
    with pytest.raises(KeyError):
        splat.chunk_workspace(acsr, torch.float16, 1, 4, 4, 1, 64)


@pytest.mark.parametrize("at", range(5))
def test_sizes_past_32_bits(acsr, at):
    args = [1, 4, 2, 8, 64]
    splat.chunk_workspace(acsr, torch.bfloat16, *args)
    args[at] += 2 ** 32
    with pytest.raises((ValueError, splat.SplatError)):
        splat.chunk_workspace(acsr, torch.bfloat16, *args)


def test_null_arguments(acsr):
    lib = splat.load()
    n = ctypes.c_int64()
    assert lib.splat_chunk_workspace(None, 0, 1, 4, 4, 1, 64, ctypes.byref(n)) == 1
    assert lib.splat_chunk_workspace(acsr.handle, 0, 1, 4, 4, 1, 64, None) == 1
    assert lib.splat_sparse_mhsa_chunk(acsr.handle, 0, 1, 1, 64, None, None, None, None, 1.0, None, None, None, None) == 1


def test_host_tensors(acsr):
    x = torch.zeros(2, 2, 8, 64)
    n = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        splat.sparse_mhsa_chunk(acsr, x, x, x, torch.zeros(2, 1, dtype=torch.int32), n, 1.0)
