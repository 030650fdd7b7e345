"""The attention weight that cached keys gather, against a plain 64-bit
implementation, and the run of a server that keeps its caches within a budget.

Bounds.  A probability p = exp(s - lse) is off by the score's error, C (A(s) + 2 +
|lse|) of it as in the chunk's tests (C = 32 * 2^-24), the given lse's own rounding
among them; sums of n rows by sqrt(n) 2^-24 at most n/32 accumulated in turn, within C
up to 2^16 rows; decay and the last sum by 2 * 2^-24 of the result.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_chunk import MASKS, TYPES, chunk64, ints, make
from test_gpu_grad import C
from test_gpu_serve import paged

pytestmark = pytest.mark.gpu


def weights64(Q, lse, kc, table, lengths, counts, M, scale, w, decay, out=None):
    """(out, its bound) in 64 bits, over a copy of w (or of out)."""
    H, heads, page = Q.shape[1], kc.shape[1], kc.shape[2]
    G = H // heads
    new, bound = (w if out is None else out).double().clone(), torch.zeros(w.shape, dtype=torch.float64)
    for b, (n, c) in enumerate(zip(lengths, counts)):
        cols = np.arange(n)
        p, o = table[b].long()[cols // page], torch.from_numpy(cols % page)
        for kh in range(heads if n else 0):
            old = w[p, kh, o].double() * (decay if c else 1.0)
            old[n - c:] = 0.0
            add, err = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
            if c:
                m = torch.from_numpy(np.ascontiguousarray(M[n - c:n, :n]))
                k = kc[p, kh, o].double()
                q = Q[b, kh * G:kh * G + G, :c].double()
                l = lse[b, kh * G:kh * G + G, :c, None].double()
                x = torch.where(m, (q @ k.t() * scale - l).exp(), 0.0)
                a = q.abs() @ k.abs().t() * abs(scale)
                add, err = x.sum((0, 1)), (x * C * (a + 2 + l.abs().nan_to_num(posinf=0.0))).sum((0, 1))
            new[p, kh, o] = old + add
            bound[p, kh, o] = err + 4 * 2.0 ** -24 * (old.abs() + add)
    return new, bound


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,H,heads", [(64, 2, 2), (128, 6, 2), (64, 5, 1), (128, 40, 1), (64, 16, 4)])
@pytest.mark.parametrize("kind,params,L", MASKS)
def test_weights(gpu_lib, kind, params, L, H, heads, d, dtype):
    splat = gpu_lib
    print(f"[gpu] weights {kind} {params} L={L} H={H},{heads} d={d} {dtype}", flush=True)
    a, M = make(splat, kind, params, L)
    g = torch.Generator().manual_seed(L + H)
    half = L // 2
    for page, T, lengths, counts in ((16, 1, [L, 1, 0, half], [1, 1, 0, 0]), (128, 7, [L, 7, half, 20], [7, 7, 3, 0]),
                                     (1, 33, [L, 40], None), (64, 150, [min(L, 290), half, 1], [min(L, 150), min(half, 131), 1])):
        T = min(T, L)
        n = counts or [T] * len(lengths)
        kc, _, table = paged(lengths, page, -(-L // page), heads, d, dtype, L)
        Q = torch.randn((len(lengths), H, T, d), generator=g).to(dtype)
        w = torch.randn(kc.shape[:3], generator=g).exp()
        scale = 1 / math.sqrt(d)
        lse = chunk64(Q, kc, kc, table, lengths, n, M, scale)[2].float()
        for decay, into in ((1.0, False), (0.75, True), (0.0, False)):
            dw = w.cuda()
            out = torch.full_like(dw, 7.0) if into else None
            r = splat.cache_weights(a, Q.cuda(), lse.cuda(), kc.cuda(), table.cuda(), ints(lengths), dw, scale,
                                    counts=None if counts is None else ints(n), decay=decay, out=out)
            torch.cuda.synchronize()
            assert r.data_ptr() == (out if into else dw).data_ptr()
            if into:
                assert torch.equal(dw.cpu(), w)
            want, bound = weights64(Q, lse, kc, table, lengths, n, M, scale, w, decay,
                                    torch.full_like(w, 7.0) if into else None)
            over = ((r.double().cpu() - want).abs() - bound).max().item()
            assert over <= 0, over


def test_new_places_start_from_zero(gpu_lib):
    """NaN weights and keys that no row has, in the chunk's own places too, do not
    reach anything; rows of lse -inf add nothing; NaN reaches its row's keys alone."""
    splat = gpu_lib
    a, M = make(splat, "window", {"w": 20}, 300)
    for T in (2, 60, 140):
        lengths, counts, page = [300, 170], [T, T - 1], 16
        kc, _, table = paged(lengths, page, 19, 2, 64, torch.float32, 3)
        Q = torch.randn((2, 4, T, 64), generator=torch.Generator().manual_seed(1))
        lse = chunk64(Q, kc, kc, table, lengths, counts, M, 0.125)[2].float()
        w = torch.rand(kc.shape[:3])
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


def test_bad_lengths_and_pages(gpu_lib):
    splat = gpu_lib
    a, M = make(splat, "full", {}, 200)
    T, lengths, counts = 5, [200, 201, -1, 4, 150, 0], [5, 5, 5, 5, 5, 0]
    kc, _, table = paged([200] * 6, 8, 25, 2, 64, torch.float32, 3)
    table[4, 2], table[4, 18] = -1, 10 ** 6
    Q, lse = torch.randn((6, 2, T, 64)), torch.full((6, 2, T), 3.0)
    w = torch.rand(kc.shape[:3])
    got = splat.cache_weights(a, Q.cuda(), lse.cuda(), kc.cuda(), table.cuda(), ints(lengths), w.cuda(), 0.125,
                              counts=ints(counts)).cpu()
    want = w.double().clone()
    for b in (0, 4):
        fixed = table.clone()
        good, bound = weights64(Q[b:b + 1], lse[b:b + 1], kc, fixed[b:b + 1].clamp(0, kc.shape[0] - 1), [lengths[b]], [5], M,
                                0.125, w, 1.0)
        for j in range(lengths[b]):
            p = int(table[b, j // 8])
            if 0 <= p < kc.shape[0]:
                assert ((got[p, :, j % 8].double() - good[p, :, j % 8]).abs() <= bound[p, :, j % 8]).all()
                want[p, :, j % 8] = got[p, :, j % 8].double()
    assert torch.equal(got.double(), want)      # nothing else was written


@pytest.mark.parametrize("dtype", TYPES)
def test_a_server_within_a_budget(gpu_lib, dtype):
    """Picture tokens turned by three axes, appended in chunks and token by token,
    attended, weighed; whenever a cache has passed its budget the lightest keys go and new
    tokens follow behind, at their own positions.  Against the same steps in 64 bits
    on the keys that the caches really hold."""
    splat = gpu_lib
    B, H, heads, d, page, L, budget = 2, 4, 2, 64, 8, 96, 40
    a, M = make(splat, "causal", {}, L)
    rot = splat.Rotary(300, 64, axes=(8, 12, 12), cyclic=True)
    g = torch.Generator().manual_seed(9)
    pages = 2 * B * (L // page)
    kc, vc = (torch.full((pages, heads, page, d), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    w = torch.full((pages, heads, page), math.nan, device="cuda")
    free = torch.randperm(pages, generator=g).int().view(2, B, L // page).cuda()
    table, side = free[0].contiguous(), 1
    n = ints([0] * B)
    seen = 0
    for step, T in enumerate((30, 25, 1, 1, 20, 1, 30, 1)):
        x = [torch.randn((B, T, h, d), generator=g).to(dtype).cuda().transpose(1, 2) for h in (H, heads, heads)]
        pos = torch.stack((torch.full((B, T), seen // 16), torch.arange(seen, seen + T).expand(B, T) // 4 % 4,
                           torch.arange(seen, seen + T).expand(B, T) % 4)).int().cuda()
        seen += T
        q = splat.cache_append(kc, vc, table, n, x[1], x[2], rot=rot, Q=x[0], positions=pos)
        want_q = splat.rotary(rot, x[0], positions=pos)
        assert torch.equal(q, want_q)
        n = n + T
        O, lse = splat.sparse_mhsa_chunk(a, q, kc, vc, table, n, 0.125)
        before = w.clone()
        splat.cache_weights(a, q, lse, kc, table, n, w, 0.125, decay=0.9)
        torch.cuda.synchronize()
        sizes = n.tolist()
        ck, cv, ct = kc.cpu(), vc.cpu(), table.cpu()
        O64, bO, l64, bl = chunk64(q.cpu(), ck, cv, ct, sizes, [T] * B, M, 0.125)
        assert ((O.double().cpu() - O64).abs() <= bO).all() and ((lse.double().cpu() - l64).abs() <= bl).all()
        want, bound = weights64(q.cpu(), lse.cpu(), ck, ct, sizes, [T] * B, M, 0.125, before.cpu(), 0.9)
        assert ((w.double().cpu() - want).abs() <= bound)[bound > 0].all()
        if max(sizes) > budget:
            to = free[side].contiguous() if step % 2 else None
            held = kc.clone(), table.clone()
            kept, n = splat.cache_evict(kc, vc, w, table, n, budget, first=2, recent=5, to=to)
            if to is not None:
                table, side = to, 1 - side
            torch.cuda.synchronize()
            assert n.tolist() == [budget] * B
            for b in range(B):
                for h in range(heads):
                    j = kept[b, h].long()
                    i = torch.arange(budget, device="cuda")
                    assert torch.equal(kc[table[b].long()[i // page], h, i % page],
                                       held[0][held[1][b].long()[j // page], h, j % page])
    assert seen == 109


def test_graph_replays(gpu_lib):
    """A step of append, chunk, weights and eviction captured once, replayed as
    sequences grow and shrink."""
    splat = gpu_lib
    B, H, heads, d, page, T, budget = 2, 4, 2, 64, 16, 3, 30
    a, _ = make(splat, "causal", {}, 64)
    kc, vc, table = (x.cuda() for x in paged([64, 64], page, 4, heads, d, torch.bfloat16, 3))
    w = torch.rand(kc.shape[:3], device="cuda")
    start, n, left = ints([20, 9]), ints([0, 0]), ints([0, 0])
    kept = torch.empty((B, heads, budget), dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn((B, h, T, d), device="cuda").bfloat16() for h in (H, heads, heads))
    qr, O, lse = torch.empty_like(q), torch.empty_like(q), torch.empty((B, H, T), device="cuda")
    rot = splat.Rotary(64, 64)
    ws = torch.empty(max(16, splat.chunk_workspace(a, torch.bfloat16, B, H, heads, T, d)), dtype=torch.uint8, device="cuda")

    def step(kc, vc, w, start, n, kept, left, qr, O, lse):
        splat.cache_append(kc, vc, table, start, k, v, rot=rot, Q=q, Qr=qr)
        torch.add(start, T, out=n)
        splat.sparse_mhsa_chunk(a, qr, kc, vc, table, n, 0.125, O=O, lse=lse, workspace=ws)
        splat.cache_weights(a, qr, lse, kc, table, n, w, 0.125, decay=0.5)
        splat.cache_evict(kc, vc, w, table, n, budget, recent=4, kept=kept, left=left)
        start.copy_(left)

    state = [kc, vc, w, start, n, kept, left, qr, O, lse]
    twin = [x.clone() for x in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*[x.clone() for x in state])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*state)
    for r in range(8):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        step(*twin)
        torch.cuda.synchronize()
        for x, y in zip(state, twin):
            assert torch.equal(x, y)
    assert start.tolist() == [30, 30]


def test_refusals(gpu_lib):
    splat = gpu_lib
    a, _ = make(splat, "window", {"w": 3}, 48)
    kc = torch.randn((6, 2, 16, 64), device="cuda")
    table = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    at = torch.full((2,), 40, dtype=torch.int32, device="cuda")
    Q, lse, w = torch.randn((2, 4, 8, 64), device="cuda"), torch.zeros((2, 4, 8), device="cuda"), torch.zeros((6, 2, 16), device="cuda")
    call = lambda **kw: splat.cache_weights(**{**dict(acsr=a, Q=Q, lse=lse, k_cache=kc, table=table, lengths=at, weights=w,
                                                      scale=1.0), **kw})
    bad = [lambda: call(Q=Q[:1]), lambda: call(Q=Q[:, :3]), lambda: call(Q=Q.bfloat16()), lambda: call(Q=Q[..., ::2]),
           lambda: call(lse=lse[:, :1]), lambda: call(lse=lse.double()), lambda: call(lengths=at.long()),
           lambda: call(counts=at[:1]), lambda: call(weights=w[:3]), lambda: call(weights=w.double()),
           lambda: call(weights=w.transpose(0, 1)), lambda: call(out=w[:3]), lambda: call(out=lse), lambda: call(decay=-0.1),
           lambda: call(decay=math.nan), lambda: call(decay=math.inf), lambda: call(out=kc.view(-1)[:192].view(6, 2, 16)),
           lambda: call(out=Q.view(-1)[:192].view(6, 2, 16)), lambda: call(k_cache=kc.bfloat16()), lambda: call(Q=Q.cpu()),
           lambda: call(table=table[:1])]
    for i, g in enumerate(bad):
        with pytest.raises((splat.SplatError, TypeError, ValueError)) as e:
            g()
        if isinstance(e.value, splat.SplatError):
            assert e.value.name in ("INVALID_ARG", "UNSUPPORTED"), (i, e.value)
    torch.cuda.synchronize()
    assert (w == 0).all()
