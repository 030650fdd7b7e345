"""Chunks that take tiles of 128 rows (bf16 launches with many units), over every mask
family: enough heads for the choice, the references on the GPU (bounds as in
test_gpu_chunk)."""
import math

import numpy as np
import pytest
import torch

from test_gpu_chunk import MASKS, check, chunk64, ints, make
from test_gpu_serve import paged

pytestmark = pytest.mark.gpu


def heads_for_tiles(splat, a, B, G, T, d):
    heads = 1
    while splat.chunk_route(a, torch.bfloat16, B, G * heads, heads, T, d)[0] != "tiles":
        heads *= 2
    return heads


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G,T,page", [(1, 150, 16), (2, 70, 64), (3, 130, 8), (5, 41, 1), (1, 260, 256), (40, 7, 4)])
@pytest.mark.parametrize("kind,params,L", MASKS)
def test_tiles(gpu_lib, kind, params, L, G, T, page, d):
    splat = gpu_lib
    a, M = make(splat, kind, params, L)
    T = min(T, L)
    heads = heads_for_tiles(splat, a, 2, G, T, d)
    print(f"[gpu] tiles {kind} {params} L={L} G={G} heads={heads} T={T} page={page} d={d}", flush=True)
    lengths, counts = [L, max(T, L // 2 + 3)], [T, T - T // 3]
    kc, vc, table = paged(lengths, page, -(-L // page), heads, d, torch.bfloat16, L)
    Q = torch.randn((2, G * heads, T, d), generator=torch.Generator().manual_seed(T)).bfloat16()
    # a few heads of all are compared, the first, the last and ones between
    some = sorted({0, heads - 1, heads // 2, heads // 3})
    q = [h * G + g for h in some for g in range(G)]
    for scale in (1 / math.sqrt(d), -0.3):
        O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths), scale,
                                         counts=ints(counts))
        torch.cuda.synchronize()
        check((O[:, q], lse[:, q]), chunk64(Q[:, q], kc[:, some], vc[:, some], table, lengths, counts, M, scale))


def test_values_that_are_not_finite(gpu_lib):
    """NaN and infinities in a newer token's key and value, a page that is none, rows
    whose scores are all -inf, in blocks that tiles take: each reaches its own rows."""
    splat, T, G, d = gpu_lib, 150, 2, 64
    a, M = make(splat, "sliding", {"w": 90, "n_global": 4}, 700)
    heads = heads_for_tiles(splat, a, 3, G, T, d)
    lengths, counts = [700, 560, 650], [T, T, T]
    kc, vc, table = paged(lengths, 16, 44, heads, d, torch.bfloat16, 3)
    Q = torch.randn((3, G * heads, T, d), generator=torch.Generator().manual_seed(1)).bfloat16()
    some, q = [0, heads - 1], [0, 1, G * heads - 2, G * heads - 1]
    want = chunk64(Q[:, q], kc[:, some], vc[:, some], table, lengths, counts, M, 0.125)
    at = lambda b, j: (int(table[b, j // 16]), slice(None), j % 16)
    k, v = kc.clone(), vc.clone()
    k[at(0, 680)], v[at(0, 680)] = math.nan, math.inf
    v[at(1, 555)] = -math.inf
    bad = table.clone()
    bad[2, 600 // 16] = -5
    O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), k.cuda(), v.cuda(), bad.cuda(), ints(lengths), 0.125)
    torch.cuda.synchronize()
    O, lse = O[:, q].double().cpu(), lse[:, q].double().cpu()
    hit = [M[550:700, 680], M[410:560, 555], M[500:650, 592:608].any(1)]
    for b in range(3):
        rows = torch.from_numpy(~hit[b])
        assert ((O[b] - want[0][b]).abs() <= want[1][b])[:, rows].all()
        assert ((lse[b] - want[2][b]).abs() <= want[3][b])[:, rows].all()
        assert not torch.isfinite(O[b][:, ~rows]).any()
    assert torch.isnan(lse[2][:, torch.from_numpy(hit[2])]).all()
    # all scores of a sequence -inf
    Q[..., 0], kc[..., 0] = 1.0, 0.0
    kc[table[1, :35].long(), :, :, 0] = -math.inf
    O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths), 0.125)
    assert torch.isnan(O[1]).all() and (lse[1] == -math.inf).all() and torch.isfinite(O[0]).all()


def test_large_scores(gpu_lib):
    """Scores of hundreds that rise and fall from tile to tile."""
    splat, T = gpu_lib, 200
    a, M = make(splat, "causal", {}, 700)
    heads = heads_for_tiles(splat, a, 1, 1, T, 64)
    for order in (1, -1):
        kc, vc, table = paged([700], 16, 44, heads, 64, torch.bfloat16, 3)
        j = torch.arange(700)
        ramp = (j if order > 0 else 699 - j).float() / 700 * 8
        kc[table[0, j // 16].long(), :, j % 16] += ramp[:, None, None].bfloat16()
        Q = (torch.randn((1, heads, T, 64), generator=torch.Generator().manual_seed(T)) + 1).bfloat16()
        for scale in (0.125, 1.0, -1.0, 0.0):
            O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints([700]), scale)
            torch.cuda.synchronize()
            check((O[:, :2], lse[:, :2]), chunk64(Q[:, :2], kc[:, :2], vc[:, :2], table, [700], [T], M, scale))
