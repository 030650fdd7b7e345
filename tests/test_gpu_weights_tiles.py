"""Weights by blocks of 64 keys (bf16 launches of many rows): new places, rows of padding,
values that are not finite, bad lengths, counts and pages (bounds as in test_gpu_weights)."""
import math

import numpy as np
import pytest
import torch

from test_gpu_chunk import MASKS, chunk64, ints, make
from test_gpu_serve import paged
from test_gpu_weights import weights64

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def tiles(splat, a, B, H, heads, T, d, room):
    assert splat.weights_route(a, BF16, B, H, heads, T, d, room)[0] == "tiles"


@pytest.mark.parametrize("d,page", [(64, 16), (128, 1), (64, 4), (128, 64)])
@pytest.mark.parametrize("G,T", [(1, 300), (5, 90), (16, 30), (3, 150)])
@pytest.mark.parametrize("kind,params,L", MASKS)
def test_masks(gpu_lib, kind, params, L, G, T, d, page):
    """Every mask family, sequences shorter and longer than the chunk, counts of every size."""
    splat, heads = gpu_lib, 2
    a, M = make(splat, kind, params, L)
    T, H = min(T, L), G * heads
    lengths, counts = [L, max(T - 5, L // 3), L // 2, 7], [T, T - 5, min(T, 33, L // 2), 0]
    if G * T >= 192:       # (rows of shorter masks than that are few, whatever the kernel)
        tiles(splat, a, 4, H, heads, T, d, -(-L // page) * page)
    print(f"[gpu] weights by tiles {kind} {params} L={L} G={G} T={T} d={d} page={page}", flush=True)
    kc, _, table = paged(lengths, page, -(-L // page), heads, d, BF16, L)
    g = torch.Generator().manual_seed(T)
    Q = torch.randn((4, H, T, d), generator=g).bfloat16()
    scale = 1 / math.sqrt(d)
    lse = chunk64(Q, kc, kc, table, lengths, counts, M, scale)[2].float()
    w = torch.randn(kc.shape[:3], generator=g).exp()
    want, bound = weights64(Q, lse, kc, table, lengths, counts, M, scale, w, 0.75)
    for b, c in enumerate(counts):
        Q[b, :, c:], lse[b, :, c:] = math.nan, math.nan        # padding is not read
    got = splat.cache_weights(a, Q.cuda(), lse.cuda(), kc.cuda(), table.cuda(), ints(lengths), w.cuda(), scale,
                              counts=ints(counts), decay=0.75)
    torch.cuda.synchronize()
    over = ((got.double().cpu() - want).abs() - bound).max().item()
    assert over <= 0, over


def test_new_places_start_from_zero(gpu_lib):
    """NaN weights and keys that no row has, in the chunk's own places too, do not
    reach anything; rows of lse -inf add nothing; NaN reaches its row's keys alone."""
    splat, page = gpu_lib, 16
    a, M = make(splat, "window", {"w": 20}, 300)
    for T, G in ((140, 4), (60, 8)):
        lengths, counts, H = [300, 170], [T, T - 1], 2 * G
        tiles(splat, a, 2, H, 2, T, 64, 304)
        kc, _, table = paged(lengths, page, 19, 2, 64, BF16, 3)
        Q = torch.randn((2, H, T, 64), generator=torch.Generator().manual_seed(1)).bfloat16()
        lse = chunk64(Q, kc, kc, table, lengths, counts, M, 0.125)[2].float()
        w = torch.rand(kc.shape[:3], generator=torch.Generator().manual_seed(2))
        want, bound = weights64(Q, lse, kc, table, lengths, counts, M, 0.125, w, 0.5)
        for b, (n, c) in enumerate(zip(lengths, counts)):
            j = np.arange(n - c, n)
            w[table[b].long()[j // page], :, j % page] = math.nan
            j = np.nonzero(~M[n - c:n, :n].any(0))[0]
            kc[table[b].long()[j // page], :, j % page] = math.nan
        run = lambda l: splat.cache_weights(a, Q.cuda(), l.cuda(), kc.cuda(), table.cuda(), ints(lengths), w.cuda(),
                                            0.125, counts=ints(counts), decay=0.5).double().cpu()
        got = run(lse)
        used = bound > 0
        assert ((got - want).abs() <= bound)[used].all()
        lse[0, 1, 0] = math.nan
        got, j = run(lse), np.arange(300)
        at = (table[0].long()[j // page], torch.from_numpy(j % page))
        assert torch.equal(torch.isnan(got[at[0], 0, at[1]]), torch.from_numpy(M[300 - T]))
        assert not torch.isnan(got[at[0], 1, at[1]]).any()
        lse[:] = -math.inf
        got = run(lse)[at[0], :, at[1]]
        assert (got[300 - T:] == 0).all() and torch.equal(got[:300 - T], (w[at[0], :, at[1]] * 0.5)[:300 - T].double())


@pytest.mark.parametrize("T,G", [(70, 8), (5, 64)])
def test_bad_lengths_and_pages(gpu_lib, T, G):
    splat, H = gpu_lib, 2 * G
    a, M = make(splat, "full", {}, 200)
    lengths, counts = [200, 201, -1, T - 1, 150, 0], [T, T, T, T, T, 0]
    tiles(splat, a, 6, H, 2, T, 64, 200)
    kc, _, table = paged([200] * 6, 8, 25, 2, 64, BF16, 3)
    table[4, 2], table[4, 18] = -1, 10 ** 6
    Q = torch.randn((6, H, T, 64), generator=torch.Generator().manual_seed(4)).bfloat16()
    lse = torch.full((6, H, T), 3.0)
    w = torch.rand(kc.shape[:3], generator=torch.Generator().manual_seed(2))
    got = splat.cache_weights(a, Q.cuda(), lse.cuda(), kc.cuda(), table.cuda(), ints(lengths), w.cuda(), 0.125,
                              counts=ints(counts)).cpu()
    want = w.double().clone()
    for b in (0, 4):
        good, bound = weights64(Q[b:b + 1], lse[b:b + 1], kc, table[b:b + 1].clamp(0, kc.shape[0] - 1), [lengths[b]], [T], M,
                                0.125, w, 1.0)
        for j in range(lengths[b]):
            p = int(table[b, j // 8])
            if 0 <= p < kc.shape[0]:
                assert ((got[p, :, j % 8].double() - good[p, :, j % 8]).abs() <= bound[p, :, j % 8]).all()
                want[p, :, j % 8] = got[p, :, j % 8].double()
    assert torch.equal(got.double(), want)      # nothing else was written
