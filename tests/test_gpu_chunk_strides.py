"""Chunks under masks of strided runs: long ones, several a row, ones that the next row's
continue and ones that they do not (bounds as in test_gpu_chunk)."""
import math

import numpy as np
import pytest
import torch

from test_gpu_chunk import TYPES, check, chunk64, ints
from test_gpu_serve import paged

pytestmark = pytest.mark.gpu


def strided(L, parts):
    """(terms, mask) of the keys c, c + s, .. up to a row's own, or up to the third number
    for rows from 1300 on."""
    i, j = np.arange(L)[:, None], np.arange(L)[None, :]
    terms, M = [], np.zeros((L, L), dtype=bool)
    for s, c, *hi in parts:
        terms.append(dict(row_lo=1300, lo_c=c, hi_c=hi[0], stride=s) if hi else dict(lo_c=c, hi_i=1, stride=s))
        M |= (j >= c) & ((j - c) % s == 0) & ((i >= 1300) & (j <= hi[0]) if hi else j <= i)
    return terms, M


PARTS = [[(2, 0)], [(3, 1)], [(31, 5)], [(32, 0)], [(33, 7)], [(64, 63)], [(501, 3)], [(7, 3, 880), (13, 1000, 1290)],
         [(2, 1, 300), (50, 350, 700), (3, 720, 1000), (1, 1100, 1111)], [(4, 2, 200), (9, 222, 2000)]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("parts", PARTS)
@pytest.mark.parametrize("T,H,heads", [(1, 4, 4), (40, 3, 1), (130, 2, 2)])
def test_strides(gpu_lib, T, H, heads, parts, dtype):
    splat, L = gpu_lib, 2900
    terms, M = strided(L, parts)
    a = splat.Acsr(splat.Pattern.from_terms(L, terms))
    print(f"[gpu] strides {parts} T={T} H={H},{heads} {dtype}", flush=True)
    lengths, counts = [L, 1501, T], [T, T - T // 3, T]
    kc, vc, table = paged(lengths, 16, -(-L // 16), heads, 64, dtype, L)
    Q = torch.randn((3, H, T, 64), generator=torch.Generator().manual_seed(T)).to(dtype)
    O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths), 0.125, counts=ints(counts))
    torch.cuda.synchronize()
    check((O, lse), chunk64(Q, kc, vc, table, lengths, counts, M, 0.125))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("w,g", [(300, 2), (200, 5), (40, 31)])
def test_residues(gpu_lib, w, g, dtype):
    """Dilated windows, whose neighbouring rows have other keys."""
    splat, L, T = gpu_lib, 1700, 131
    a = splat.Acsr(splat.Pattern.dilated(L, w, g))
    i, j = np.arange(L)[:, None], np.arange(L)[None, :]
    M = ((j - i) % g == 0) & (np.abs(j - i) <= g * w)
    lengths, counts = [L, 1000], [T, 77]
    for page in (1, 64):
        kc, vc, table = paged(lengths, page, -(-L // page), 2, 64, dtype, L)
        Q = torch.randn((2, 4, T, 64), generator=torch.Generator().manual_seed(T)).to(dtype)
        O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths), 0.125, counts=ints(counts))
        torch.cuda.synchronize()
        check((O, lse), chunk64(Q, kc, vc, table, lengths, counts, M, 0.125))
