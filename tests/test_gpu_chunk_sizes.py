"""Chunks, weights and eviction at the ends of their ranges: 65536 positions, caches
past 2^32 bytes, more than 64 sequences, every page size and head layout, against plain
64-bit implementations (bounds as in test_gpu_chunk and test_gpu_weights)."""
import math

import numpy as np
import pytest
import torch

from test_gpu_chunk import check, chunk64, ints, make
from test_gpu_evict import evicted, same, setup
from test_gpu_grad import C, HALF
from test_gpu_serve import paged
from test_gpu_weights import weights64

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]


def both(splat, a, M, Q, kc, vc, table, lengths, counts, scale, device="cpu"):
    """A chunk and its weights, against 64 bits."""
    d = [x.cuda() for x in (Q, kc, vc, table)]
    O, lse = splat.sparse_mhsa_chunk(a, *d, ints(lengths), scale, counts=ints(counts))
    w = torch.rand(kc.shape[:3], generator=torch.Generator().manual_seed(1))
    got = splat.cache_weights(a, d[0], lse, d[1], d[3], ints(lengths), w.cuda(), scale, counts=ints(counts), decay=0.5)
    torch.cuda.synchronize()
    check((O, lse), chunk64(Q, kc, vc, table, lengths, counts, M, scale, device=device))
    want, bound = weights64(Q, lse.cpu(), kc, table, lengths, counts, M, scale, w, 0.5)
    assert ((got.double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [1, 2, 4, 8, 16, 32, 64])
@pytest.mark.parametrize("T", [3, 50, 140])
def test_page_sizes(gpu_lib, T, page, dtype):
    splat = gpu_lib
    a, M = make(splat, "sliding", {"w": 70, "n_global": 5}, 420)
    lengths, counts = [420, 401, 150], [T, T - 1, min(T, 150)]
    for d, H, heads in ((64, 3, 3), (128, 4, 2)):
        kc, vc, table = paged(lengths, page, -(-420 // page), heads, d, dtype, page)
        Q = torch.randn((3, H, T, d), generator=torch.Generator().manual_seed(T)).to(dtype)
        both(gpu_lib, a, M, Q, kc, vc, table, lengths, counts, 1 / math.sqrt(d))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,heads", [(3, 1), (7, 7), (96, 2), (130, 1), (200, 2)])
@pytest.mark.parametrize("T", [1, 2, 30])
def test_head_layouts(gpu_lib, T, H, heads, dtype):
    """Groups that divide no block of rows, and ones of more heads than a block's rows."""
    a, M = make(gpu_lib, "causal", {}, 200)
    kc, vc, table = paged([200, 61], 16, 13, heads, 64, dtype, 3)
    Q = torch.randn((2, H, T, 64), generator=torch.Generator().manual_seed(T)).to(dtype)
    both(gpu_lib, a, M, Q, kc, vc, table, [200, 61], [T, max(T - 7, 0)], 0.125)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,T,L", [(64, 2, 700), (65, 1, 2100), (130, 3, 900), (70, 70, 300)])
def test_many_sequences(gpu_lib, B, T, L, dtype):
    """Past the 64 sequences that a wavefront deals with at once."""
    a, M = make(gpu_lib, "causal", {}, L)
    lengths = [(L * (b + 1)) // B if b % 5 else min(b, T) for b in range(B)]
    lengths[-1] = L
    counts = [min(T, n) for n in lengths]
    kc, vc, table = paged(lengths, 16, -(-L // 16), 1, 64, dtype, 3)
    Q = torch.randn((B, 2, T, 64), generator=torch.Generator().manual_seed(T)).to(dtype)
    both(gpu_lib, a, M, Q, kc, vc, table, lengths, counts, 0.125)


@pytest.mark.parametrize("T", [17, 257])
def test_most_blocks(gpu_lib, T):
    """16384 heads of sequences that may have 65536 keys each: more blocks of keys than
    a grid's first dimension takes in threads."""
    splat, L, B, heads, page, scale = gpu_lib, 65536, 1024, 16, 512, 0.125
    a = splat.Acsr(splat.Pattern.from_terms(L, [dict(lo_i=1, lo_c=-40, hi_i=1)]))
    g = torch.Generator(device="cuda").manual_seed(T)
    kc, vc = (torch.randn((B, heads, page, 64), generator=g, device="cuda").bfloat16() for _ in range(2))
    Q = torch.randn((B, heads, T, 64), generator=g, device="cuda").bfloat16()
    table = torch.zeros((B, L // page), dtype=torch.int32)
    table[:, 0] = torch.randperm(B, generator=torch.Generator().manual_seed(1)).int()
    lengths = [T + (37 * b) % (page - T) for b in range(B)]
    w = torch.rand((B, heads, page), generator=g, device="cuda")
    O, lse = splat.sparse_mhsa_chunk(a, Q, kc, vc, table.cuda(), ints(lengths), scale)
    got = splat.cache_weights(a, Q, lse, kc, table.cuda(), ints(lengths), w, scale, decay=0.5, out=torch.empty_like(w))
    torch.cuda.synchronize()
    M = Rows(lambda i, j: (j <= i) & (j >= i - 40))
    some = [0, 1, 511, 512, 1022, 1023]
    at = table[some, 0].long()
    one = torch.arange(len(some), dtype=torch.int32)[:, None]
    n, c = [lengths[b] for b in some], [T] * len(some)
    small = [x[at.cuda()].cpu() for x in (kc, vc, w, got)]
    q, l = Q[some].cpu(), lse[some].cpu()
    check((O[some], l), chunk64(q, *small[:2], one, n, c, M, scale))
    want, bound = weights64(q, l, small[0], one, n, c, M, scale, small[2], 0.5)
    for k, length in enumerate(n):
        assert ((small[3][k].double() - want[k]).abs() <= bound[k])[:, :length].all()


class Rows:
    """Rows of a mask of 65536 positions, as chunk64 asks for them."""

    def __init__(self, rows):
        self.rows = rows

    def __getitem__(self, at):
        rows, cols = at
        i = np.arange(rows.start, rows.stop)[:, None]
        return self.rows(i, np.arange(cols.stop)[None, :])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["causal", "strided", "even"])
@pytest.mark.parametrize("T", [3, 80])
def test_65536_positions(gpu_lib, T, kind, dtype):
    splat, L = gpu_lib, 65536
    term = {"causal": [dict(hi_i=1)], "strided": [dict(lo_i=1, lo_c=-90, hi_i=1), dict(lo_c=31, hi_i=1, stride=64)],
            "even": [dict(hi_i=1, stride=2)]}[kind]
    M = Rows({"causal": lambda i, j: j <= i, "strided": lambda i, j: (j <= i) & ((j >= i - 90) | (j % 64 == 31)),
              "even": lambda i, j: (j <= i) & (j % 2 == 0)}[kind])
    lengths, counts = [L, 40001], [T, T - 1]
    # the rows that are asked for: a whole causal mask has more non-zeros than a handle takes
    term = [dict(t, row_lo=n - 100, row_hi=n) for t in term for n in lengths]
    a = splat.Acsr(splat.Pattern.from_terms(L, term))
    g = torch.Generator().manual_seed(T)
    pages = 2 * L // 256 + 3
    kc, vc = (torch.randn((pages, 1, 256, 64), generator=g).to(dtype) for _ in range(2))
    table = torch.randperm(pages, generator=g).int()[:2 * L // 256].view(2, L // 256).contiguous()
    Q = torch.randn((2, 1, T, 64), generator=g).to(dtype)
    O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths), 0.125, counts=ints(counts))
    torch.cuda.synchronize()
    # a sum's parts hold up to 2^16 / 4 terms in turn: C for 256 of them grows by sqrt(64)
    want = list(chunk64(Q, kc, vc, table, lengths, counts, M, 0.125, device="cuda"))
    want[1], want[3] = want[1] + 7 * C * want[0].abs().clamp(min=1.0), want[3] * 8
    check((O, lse), want)
    w = torch.rand(kc.shape[:3], generator=g)
    got = splat.cache_weights(a, Q.cuda(), lse, kc.cuda(), table.cuda(), ints(lengths), w.cuda(), 0.125, counts=ints(counts))
    torch.cuda.synchronize()
    full, bound = weights64(Q, lse.cpu(), kc, table, lengths, counts, M, 0.125, w, 1.0)
    assert ((got.double().cpu() - full).abs() <= bound).all()


def test_caches_past_32_bits(gpu_lib):
    """K and V of 5 GB each, the sequences' pages at their ends: chunk, weights and
    both kinds of eviction."""
    splat, heads, page, d, L = gpu_lib, 8, 64, 128, 640
    pages = 41000
    a, M = make(splat, "causal", {}, L)
    used = torch.cat((torch.arange(pages - 24, pages), torch.tensor([0, 1, 5, 7]))).int()
    order = used[torch.randperm(28, generator=torch.Generator().manual_seed(1))]
    table, to = order[:20].view(2, 10).contiguous(), order[20:28].view(2, 4).contiguous()
    lengths = [640, 500]
    small = [torch.randn((28, heads, page, d), generator=torch.Generator().manual_seed(k)).bfloat16() for k in range(2)]
    big = [torch.zeros((pages, heads, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert big[0].nbytes > 2 ** 32
    w = torch.zeros((pages, heads, page), device="cuda")
    at = {int(p): k for k, p in enumerate(used)}
    low = lambda t: torch.tensor([[at[int(p)] for p in r] for r in t], dtype=torch.int32)
    for x, y in zip(big, small):
        x[used.long().cuda()] = y.cuda()
    for T in (3, 90):
        Q = torch.randn((2, 16, T, d), generator=torch.Generator().manual_seed(T)).bfloat16()
        O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), *big, table.cuda(), ints(lengths), 0.09)
        splat.cache_weights(a, Q.cuda(), lse, big[0], table.cuda(), ints(lengths), w, 0.09)
        torch.cuda.synchronize()
        check((O, lse), chunk64(Q, *small, low(table), lengths, [T, T], M, 0.09))
    ws = w[used.long().cuda()].cpu()
    for moves in (True, False):
        want = evicted(*small, ws, low(table), low(to) if moves else None, lengths, 250, 3, 20)
        kept, left = splat.cache_evict(*big, w, table.cuda(), ints(lengths), 250, first=3, recent=20,
                                       to=to.cuda() if moves else None)
        torch.cuda.synchronize()
        got = [x[used.long().cuda()].cpu() for x in (*big, w)] + [kept, left]
        for x, y in zip(got, want):
            assert same(x, y)
        small, ws = list(want[:2]), want[2]


@pytest.mark.parametrize("dtype", TYPES)
def test_without_anything_new(gpu_lib, dtype):
    """No count at all: O = 0, weights kept undecayed."""
    splat = gpu_lib
    a, _ = make(splat, "causal", {}, 100)
    for T in (1, 80):
        kc, vc, table = (x.cuda() for x in paged([100, 3], 16, 7, 2, 64, dtype, 3))
        Q = torch.randn((2, 4, T, 64), device="cuda").to(dtype)
        O, lse = splat.sparse_mhsa_chunk(a, Q, kc, vc, table, ints([100, 3]), 0.125, counts=ints([0, 0]))
        assert (O == 0).all() and (lse == -math.inf).all()
        w = torch.rand(kc.shape[:3], device="cuda")
        before = w.clone()
        splat.cache_weights(a, Q, lse, kc, table, ints([100, 3]), w, 0.125, counts=ints([0, 0]), decay=0.5)
        assert torch.equal(w, before)
