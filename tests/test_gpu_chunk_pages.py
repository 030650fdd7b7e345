"""Caches that have given up the pages that no row of the chunk needs, as a server with a
sliding window does: a page that is none concerns the rows that have a key there and no
others, which come out bit for bit as with every page present."""
import math

import numpy as np
import pytest
import torch

from test_gpu_chunk import check, chunk64, ints, make
from test_gpu_chunk_tiles import heads_for_tiles
from test_gpu_serve import paged

pytestmark = pytest.mark.gpu


def freed(table, lengths, counts, M, page):
    """The table without the pages that no row has a key in."""
    out = table.clone()
    for b, (n, c) in enumerate(zip(lengths, counts)):
        used = np.zeros(table.shape[1], dtype=bool)
        used[np.nonzero(M[n - c:n, :n].any(0))[0] // page] = True
        out[b, torch.from_numpy(~used)] = -1
    return out


@pytest.mark.parametrize("tiles", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32, 64])
@pytest.mark.parametrize("kind,params,L,T,lengths", [("sliding", {"w": 70, "n_global": 4}, 900, 200, [893, 611, 900]),
                                                     ("window", {"w": 45}, 900, 131, [901 - 64, 450, 131]),
                                                     ("dilated", {"w": 30, "dilation": 3}, 900, 150, [877, 600, 450]),
                                                     ("strided_local", {"local": 9, "stride": 80}, 1300, 40, [1300, 1211, 700])])
def test_pages_behind_the_window(gpu_lib, kind, params, L, T, lengths, page, d, tiles):
    splat = gpu_lib
    a, M = make(splat, kind, params, L)
    heads = heads_for_tiles(splat, a, 3, 1, T, d) if tiles else 1
    assert (splat.chunk_route(a, torch.bfloat16, 3, heads, heads, T, d)[0] == "tiles") == tiles
    print(f"[gpu] freed pages {kind} page={page} d={d} tiles={tiles} heads={heads}", flush=True)
    counts = [T, T - 7, T]
    kc, vc, table = (x.cuda() for x in paged(lengths, page, -(-L // page), heads, d, torch.bfloat16, L))
    Q = torch.randn((3, heads, T, d), generator=torch.Generator().manual_seed(T)).bfloat16().cuda()
    run = lambda t: splat.sparse_mhsa_chunk(a, Q, kc, vc, t, ints(lengths), 1 / math.sqrt(d), counts=ints(counts))
    want = run(table)
    few = freed(table, lengths, counts, M, page)
    assert kind == "strided_local" or (few[0] < 0).sum() > (table[0] < 0).sum()
    got = run(few)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("page", [1, 8, 16, 64])
@pytest.mark.parametrize("G,T", [(1, 200), (3, 90)])
def test_a_page_that_some_rows_need(gpu_lib, G, T, page):
    """... NaN in the rows that have a key there, in the others no bit changes."""
    splat, L, d, spared = gpu_lib, 900, 64, False
    for kind, params in (("sliding", {"w": 70, "n_global": 4}), ("dilated", {"w": 30, "dilation": 3})):
        a, M = make(splat, kind, params, L)
        heads = heads_for_tiles(splat, a, 2, G, T, d)
        lengths = [893, 640]
        kc, vc, table = paged(lengths, page, -(-L // page), heads, d, torch.bfloat16, L)
        Q = torch.randn((2, G * heads, T, d), generator=torch.Generator().manual_seed(T)).bfloat16()
        run = lambda t: splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), t.cuda(), ints(lengths), 0.125)
        want = run(table)
        bad = freed(table, lengths, [T, T], M, page)
        hit = [np.zeros(T, dtype=bool) for _ in lengths]
        for b, j, none in ((0, 893 - T // 2, -1), (0, 893 - 20, 10 ** 6), (1, 640 - T, -2 ** 31)):
            bad[b, j // page] = none
            hit[b] |= M[lengths[b] - T:lengths[b], j // page * page:min((j // page + 1) * page, lengths[b])].any(1)
        O, lse = run(bad)
        torch.cuda.synchronize()
        for b in range(2):
            rows = torch.from_numpy(hit[b]).cuda()
            assert rows.any()
            spared = spared or not rows.all()
            assert torch.isnan(O[b][:, rows]).all() and torch.isnan(lse[b][:, rows]).all()
            assert torch.equal(O[b][:, ~rows], want[0][b][:, ~rows])
            assert torch.equal(lse[b][:, ~rows], want[1][b][:, ~rows])
    assert spared


def test_pages_given_up_in_many_parts(gpu_lib):
    """... where workgroups share out a block's keys."""
    splat, L, d, page = gpu_lib, 3000, 128, 16
    a, M = make(splat, "sliding", {"w": 1500, "n_global": 4}, L)
    T, lengths = 200, [2990]
    heads = heads_for_tiles(splat, a, 1, 1, T, d)
    assert splat.chunk_route(a, torch.bfloat16, 1, heads, heads, T, d)[1] > 1
    kc, vc, table = paged(lengths, page, -(-L // page), heads, d, torch.bfloat16, L)
    Q = torch.randn((1, heads, T, d), generator=torch.Generator().manual_seed(T)).bfloat16()
    run = lambda t: splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), t.cuda(), ints(lengths), 0.09)
    want = run(table)
    few = freed(table, lengths, [T], M, page)
    assert (few[0] < 0).sum() > 70
    got = run(few)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    few[0, (2990 - T - 700) // page] = -1
    O, lse = run(few)
    torch.cuda.synchronize()
    j = (2990 - T - 700) // page * page
    rows = torch.from_numpy(M[2990 - T:2990, j:j + page].any(1)).cuda()
    assert torch.isnan(O[0][:, rows]).all() and torch.equal(O[0][:, ~rows], want[0][0][:, ~rows])
    check((want[0][:, :2], want[1][:, :2]), chunk64(Q[:, :2], kc[:, :2], vc[:, :2], table, lengths, [T], M, 0.09))


@pytest.mark.parametrize("tiles", [True, False])
@pytest.mark.parametrize("page", [2, 16, 64])
def test_unused_pages_hold_anything(gpu_lib, page, tiles):
    """... NaN and infinities in the pages given up, the cache's first among them."""
    splat, L, d = gpu_lib, 900, 64
    for kind, params, T, lengths in (("sliding", {"w": 70, "n_global": 4}, 200, [893, 611]), ("dilated", {"w": 30, "dilation": 3}, 150, [877, 600])):
        a, M = make(splat, kind, params, L)
        heads = heads_for_tiles(splat, a, 2, 1, T, d) if tiles else 2
        kc, vc, table = paged(lengths, page, -(-L // page), heads, d, torch.bfloat16, L)
        Q = torch.randn((2, heads, T, d), generator=torch.Generator().manual_seed(T)).bfloat16()
        run = lambda k, v, t: splat.sparse_mhsa_chunk(a, Q.cuda(), k.cuda(), v.cuda(), t.cuda(), ints(lengths), 0.125)
        want = run(kc, vc, table)
        few = freed(table, lengths, [T, T], M, page)
        # a page given up becomes the cache's first
        gone = int(table[0][(few[0] < 0) & (table[0] >= 0)][0])
        swap = torch.arange(kc.shape[0])
        swap[0], swap[gone] = gone, 0
        few = torch.where(few >= 0, swap.int()[few.clamp(min=0).long()], few)
        k, v = kc[swap].clone(), vc[swap].clone()
        unused = torch.ones(k.shape[0], dtype=torch.bool)
        unused[few[few >= 0].long()] = False
        assert unused[0]
        k[unused], v[unused] = math.nan, math.inf
        got = run(k, v, few)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
