"""How a chunk's launch is sized: by its rows, not by the mask's longest.  CPU only."""
import pytest
import torch

import paper_2407_16847_amd as splat

BF16, F32 = torch.bfloat16, torch.float32


def sliding(L, w, first=4):
    return splat.Acsr(splat.Pattern.from_terms(L, [dict(lo_i=1, lo_c=-w, hi_i=1), dict(row_lo=first, hi_c=first - 1)]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,H,heads,T", [(1, 16, 16, 1), (1, 16, 16, 8), (2, 12, 12, 300), (1, 12, 12, 64), (4, 32, 8, 300),
                                         (7, 16, 2, 2), (3, 4, 4, 910), (70, 8, 8, 3)])
def test_global_rows(B, H, heads, T, d, dtype):
    """A few rows that see every key change nothing for a chunk of the others."""
    for L, w, n in ((4096, 255, 4), (4096, 512, 64), (8192, 40, 9)):
        few = [dict(lo_i=1, lo_c=-w, hi_i=1), dict(row_lo=n, hi_c=n - 1)]
        with_rows = splat.Acsr(splat.Pattern.from_terms(L, few + [dict(row_hi=n, hi_c=L - 1)]))
        without = splat.Acsr(splat.Pattern.from_terms(L, few))
        got, want = (splat.chunk_route(a, dtype, B, H, heads, T, d) for a in (with_rows, without))
        assert got == want, (L, w, n)
        assert (splat.chunk_workspace(with_rows, dtype, B, H, heads, T, d)
                == splat.chunk_workspace(without, dtype, B, H, heads, T, d))


def test_newer_keys():
    """A symmetric window's newer half counts as far as the chunk has newer tokens."""
    both = splat.Acsr(splat.Pattern.window_global(4096, 512, 64))
    past = sliding(4096, 512, 64)
    for T in (1, 2, 8, 16):
        assert splat.chunk_route(both, BF16, 1, 16, 16, T, 64) == splat.chunk_route(past, BF16, 1, 16, 16, T, 64)
    assert splat.chunk_route(both, F32, 1, 4, 4, 31, 64)[1] <= splat.chunk_route(sliding(4096, 1088, 64), F32, 1, 4, 4, 31, 64)[1]


def test_rows_that_grow():
    """Rows of every length up to the longest: the longest counts, a chunk's are the last."""
    every = splat.Acsr(splat.Pattern.from_terms(4096, [dict(hi_i=1)]))
    full = splat.Acsr(splat.Pattern.full(4096))
    for B, H, heads, T, d in ((1, 8, 8, 4, 64), (2, 12, 12, 70, 128), (16, 32, 8, 5, 128), (4, 32, 8, 1024, 128)):
        for dtype in (BF16, F32):
            assert splat.chunk_route(every, dtype, B, H, heads, T, d) == splat.chunk_route(full, dtype, B, H, heads, T, d)


def test_rows_without_keys():
    """Masks whose rows have no keys, or few rows any."""
    none = splat.Acsr(splat.Pattern.from_terms(500, [dict(row_lo=0, row_hi=1, lo_c=499, hi_c=499)]))
    assert splat.chunk_route(none, F32, 1, 4, 4, 8, 64) == ("slices", 1)
    some = splat.Acsr(splat.Pattern.from_terms(4096, [dict(row_lo=4000, row_hi=4090, hi_i=1)]))
    assert splat.chunk_route(some, F32, 1, 4, 4, 8, 64)[1] >= 16


def test_faster_side():
    """Measured launches on both sides of the choices, and how few blocks are shared out."""
    for w, L, B, H, heads, T, d, tiles in (
            (15, 2048, 6, 16, 2, 328, 64, True), (15, 2048, 2, 12, 12, 1000, 64, False), (400, 2048, 6, 12, 12, 300, 64, False),
            (200, 2048, 4, 32, 8, 300, 64, True), (1000, 4096, 2, 16, 16, 400, 64, False), (3500, 4096, 2, 16, 16, 400, 64, True),
            (15, 2048, 6, 16, 2, 328, 128, True), (63, 2048, 2, 12, 12, 1000, 128, True), (200, 2048, 6, 16, 2, 150, 128, False),
            (1000, 4096, 2, 16, 16, 400, 128, False), (1800, 4096, 2, 16, 16, 400, 128, True), (1800, 4096, 2, 12, 12, 64, 128, False)):
        route = splat.chunk_route(sliding(L, w), BF16, B, H, heads, T, d)[0]
        assert route == ("tiles" if tiles else "slices"), (w, B, H, T, d)
    for w, dtype, d, parts in ((560, BF16, 64, 5), (400, BF16, 64, 1), (160, BF16, 64, 1), (560, F32, 64, 5), (400, F32, 64, 4),
                               (160, F32, 64, 1), (160, F32, 128, 2), (64, F32, 128, 1)):
        assert splat.chunk_route(sliding(4096, w), dtype, 1, 16, 16, 8, d)[1] == parts, (w, dtype, d)
    assert splat.chunk_route(sliding(2048, 255), F32, 2, 12, 12, 300, 64) == ("slices", 1)
