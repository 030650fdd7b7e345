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


def test_route():
    """The faster side of measured launches."""
    window = splat.Acsr(splat.Pattern.from_terms(2048, [dict(lo_i=1, lo_c=-255, hi_i=1), dict(row_lo=4, hi_c=3)]))
    every = splat.Acsr(splat.Pattern.from_terms(4096, [dict(hi_i=1)]))
    bf16 = torch.bfloat16
    for acsr, B, H, heads, T, d, tiles in (
            (window, 2, 12, 12, 300, 64, False), (window, 4, 16, 16, 300, 64, False),
            (window, 4, 32, 8, 300, 64, True), (window, 4, 16, 16, 1000, 64, True), (every, 2, 12, 12, 300, 64, True),
            (window, 2, 12, 12, 300, 128, False), (window, 2, 12, 12, 1000, 128, True), (every, 2, 12, 12, 70, 128, True),
            (every, 16, 32, 8, 5, 128, False), (every, 4, 32, 8, 1024, 128, True)):
        assert splat.chunk_route(acsr, bf16, B, H, heads, T, d)[0] == ("tiles" if tiles else "slices"), (B, H, T, d)
        assert splat.chunk_route(acsr, torch.float32, B, H, heads, T, d)[0] == "slices"
    assert splat.chunk_route(every, bf16, 1, 8, 8, 4, 64)[1] > 1
    assert splat.chunk_route(every, bf16, 64, 16, 16, 64, 64)[1] == 1
    with pytest.raises(splat.SplatError):
        splat.chunk_route(every, bf16, 1, 8, 3, 4, 64)
    assert splat.load().splat_debug_chunk(every.handle, 0, 1, 8, 8, 4, 64, None) == 1
