"""The most rows that a chunk's calls take, B*H*T = 2^24, and one token more."""
import math

import pytest
import torch

from test_gpu_chunk import check, chunk64, ints, make
from test_gpu_serve import paged
from test_gpu_weights import weights64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,H,heads,T", [(16, 64, 8, 16384), (1, 32, 32, 1 << 19)])
def test_most_rows(gpu_lib, B, H, heads, T):
    splat, d, L = gpu_lib, 64, 300
    assert B * H * T == 1 << 24
    a, M = make(splat, "sliding", {"w": 40, "n_global": 4}, L)
    lengths, counts = [L - 7 * b for b in range(B)], [200 - 11 * b for b in range(B)]
    kc, vc, table = paged(lengths, 16, 19, heads, d, torch.bfloat16, 3)
    few = torch.randn((B, H, 200, d), generator=torch.Generator().manual_seed(1)).bfloat16()
    Q = torch.full((B, H, T + 1, d), math.nan, dtype=torch.bfloat16, device="cuda")       # padding: not read
    Q[:, :, :200] = few.cuda()
    dev = [x.cuda() for x in (kc, vc, table)]
    O, lse = splat.sparse_mhsa_chunk(a, Q[:, :, :T], *dev, ints(lengths), 0.125, counts=ints(counts))
    w = torch.rand(kc.shape[:3], generator=torch.Generator().manual_seed(2))
    got = splat.cache_weights(a, Q[:, :, :T], lse, dev[0], dev[2], ints(lengths), w.cuda(), 0.125, counts=ints(counts), decay=0.5)
    torch.cuda.synchronize()
    assert not O[:, :, 200:].any() and (lse[:, :, 200:] == -math.inf).all()
    small = lse[:, :, :200].cpu()
    check((O[:, :, :200], small), chunk64(few, kc, vc, table, lengths, counts, M, 0.125))
    want, bound = weights64(few, small, kc, table, lengths, counts, M, 0.125, w, 0.5)
    assert ((got.double().cpu() - want).abs() <= bound).all()
    # a token more
    more = torch.empty((B, H, T + 1), device="cuda")
    for call in (lambda: splat.sparse_mhsa_chunk(a, Q, *dev, ints(lengths), 0.125, counts=ints(counts)),
                 lambda: splat.cache_weights(a, Q, more, dev[0], dev[2], ints(lengths), w.cuda(), 0.125, counts=ints(counts))):
        with pytest.raises(splat.SplatError) as e:
            call()
        assert e.value.name == "UNSUPPORTED" and "2^24" in str(e.value)
