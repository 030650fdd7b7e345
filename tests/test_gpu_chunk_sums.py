"""Blocks of many bf16 rows divide O by the sum of the weights that met V, rounded as
they were, so that the roundings of a row's weights cancel in what its values share.

With weights w (1 + e), |e| <= 2^-8 (half a step of bf16), the result is off by
sum w e (v - O) / (1 + sum w e): at most 2^-8 / (1 - 2^-8) of sum w |v - O|, beside the
bounds of test_gpu_chunk for scores and sums (C of the terms' magnitudes) and O's own
rounding.  Where all values of a feature are one number that leaves C, so O is the number.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_chunk import chunk64, ints, make
from test_gpu_chunk_tiles import heads_for_tiles
from test_gpu_grad import C, HALF
from test_gpu_serve import paged

pytestmark = pytest.mark.gpu

CASES = [("causal", {}, 700, 1, 200, 16), ("causal", {}, 700, 3, 100, 4), ("sliding", {"w": 300, "n_global": 4}, 900, 1, 260, 64),
         ("dilated", {"w": 100, "dilation": 3}, 700, 2, 70, 8), ("full", {}, 2500, 4, 33, 64)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,params,L,G,T,page", CASES)
def test_equal_values(gpu_lib, kind, params, L, G, T, page, d):
    splat = gpu_lib
    a, _ = make(splat, kind, params, L)
    heads = heads_for_tiles(splat, a, 2, G, T, d)
    parts = splat.chunk_route(a, torch.bfloat16, 2, G * heads, heads, T, d)[1]
    print(f"[gpu] equal values {kind} L={L} G={G} T={T} d={d} parts={parts}", flush=True)
    lengths = [L, L // 2 + 5]
    kc, vc, table = paged(lengths, page, -(-L // page), heads, d, torch.bfloat16, L)
    g = torch.Generator().manual_seed(d + T)
    value = (torch.randn(d, generator=g) * 3).bfloat16()
    vc[:] = value
    Q = torch.randn((2, G * heads, T, d), generator=g).bfloat16()
    for scale in (1 / math.sqrt(d), 4 / math.sqrt(d), -0.5):
        O, _ = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths), scale)
        torch.cuda.synchronize()
        off = (O.cpu() != value).sum().item()
        assert off == 0, f"{off} of {O.numel()}"


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,params,L,G,T,page", CASES)
def test_values_far_from_zero(gpu_lib, kind, params, L, G, T, page, d):
    splat = gpu_lib
    a, M = make(splat, kind, params, L)
    heads = heads_for_tiles(splat, a, 1, G, T, d)
    print(f"[gpu] values far from zero {kind} L={L} G={G} T={T} d={d}", flush=True)
    kc, vc, table = paged([L], page, -(-L // page), heads, d, torch.bfloat16, L)
    vc = (4 + vc.float() / 16).bfloat16()
    Q = torch.randn((1, G * heads, T, d), generator=torch.Generator().manual_seed(T)).bfloat16()
    some = sorted({0, heads - 1, heads // 2})
    q = [h * G + g for h in some for g in range(G)]
    scale = 4 / math.sqrt(d)
    O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints([L]), scale)
    torch.cuda.synchronize()
    want, _, l64, lbound = chunk64(Q[:, q], kc[:, some], vc[:, some], table, [L], [T], M, scale)
    assert ((lse[:, q].double().cpu() - l64).abs() <= lbound).all()
    j = np.arange(L)
    p, o = table[0].long()[j // page], torch.from_numpy(j % page)
    m = torch.from_numpy(np.ascontiguousarray(M[L - T:]))
    half = HALF[torch.bfloat16]
    for i, h in enumerate(q):
        k, v = (x[p, h // G, o].double() for x in (kc, vc))
        s = (Q[0, h].double() @ k.t() * scale).masked_fill(~m, -math.inf)
        A = Q[0, h].double().abs() @ k.t().abs() * scale
        w = torch.softmax(s, -1)
        ref = want[0, i]
        err = w * C * (2 + A + (w * A).sum(-1, keepdim=True))
        spread = torch.stack([(w * (v[:, f] - ref[:, f, None]).abs()).sum(-1) for f in range(d)], -1)
        bound = spread * half / (1 - half) + (err @ v.abs()) + half * ref.abs()
        over = ((O[0, h].double().cpu() - ref).abs() - bound).max().item()
        assert over <= 0, (h, over)
