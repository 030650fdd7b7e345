"""Rotary positions, the paged cache and the attention of single query tokens
over it, against plain 64-bit implementations.

Bounds.  The rotation: two fp32 products and their sum of inputs within 2^-24 of
exact angles' cosines and sines, 4 * 2^-24 of |x| + |y| of the pair, and one
rounding to bf16 (2^-8 of the result).  The attention: C = 32 * 2^-24 of the
terms' magnitudes as in the training tests, P held as two bf16 parts beside a
bf16 V (2^-16 of it), and one rounding to bf16.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_grad import C, HALF, make
from test_host_serve import frequencies

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]


def rotate64(x, pos, R, inter, inverse=False, magnitude=1.0, **kw):
    """(x [B, H, T, d] turned to pos [B, T], the sum of a pair's magnitudes)."""
    x = x.double()
    a = pos.double()[:, None, :, None] * torch.from_numpy(frequencies(R, **kw))
    c, s = a.cos() * magnitude, a.sin() * magnitude * (-1 if inverse else 1)
    first, second = (slice(0, R, 2), slice(1, R, 2)) if inter else (slice(0, R // 2), slice(R // 2, R))
    p, q = x[..., first], x[..., second]
    y, m = x.clone(), torch.zeros_like(x)
    y[..., first], y[..., second] = p * c - q * s, q * c + p * s
    m[..., first] = m[..., second] = (p.abs() + q.abs()) * magnitude
    return y, m


def rotary_check(name, got, x, pos, **kw):
    want, m = rotate64(x, pos, **kw)
    got = got.double().cpu()
    over = ((got - want).abs() - 4 * 2.0 ** -24 * m - HALF[x.dtype] * want.abs()).max().item()
    assert over <= 0, f"{name}: {over}"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,R", [(64, 16), (64, 64), (128, 32), (128, 96), (128, 128)])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("B,H,H2,T", [(1, 1, 1, 1), (2, 3, 1, 37), (3, 40, 8, 65), (2, 5, 5, 1000)])
def test_rotary(gpu_lib, B, H, H2, T, inter, d, R, dtype):
    splat = gpu_lib
    print(f"[gpu] rotary B={B} H={H},{H2} T={T} d={d} R={R} {inter} {dtype}", flush=True)
    g = torch.Generator().manual_seed(T + R)
    rot = splat.Rotary(70000, R, interleaved=inter)
    q = torch.randn((B, T, H, d), generator=g).to(dtype).transpose(1, 2)
    k = torch.randn((B, H2, T, d), generator=g).to(dtype)
    pos = torch.randint(0, 70000, (B, T), generator=g, dtype=torch.int32)
    here = torch.arange(T, dtype=torch.int32).expand(B, T)
    kw = dict(R=R, inter=inter)
    for p, at in ((None, here), (pos.cuda(), pos)):
        for inverse in (False, True):
            yq, yk = splat.rotary(rot, q.cuda(), k.cuda(), positions=p, inverse=inverse)
            one = splat.rotary(rot, k.cuda(), positions=p, inverse=inverse)
            torch.cuda.synchronize()
            assert yq.is_contiguous() and yq.dtype == dtype and torch.equal(one, yk)
            rotary_check("q", yq, q, at, inverse=inverse, **kw)
            rotary_check("k", yk, k, at, inverse=inverse, **kw)
    # in place, in a joint buffer of Q, K and V, of which V stays as it was
    if H == H2:
        qkv = torch.randn((B, T, 3, H, d), generator=g).to(dtype)
        dev = qkv.cuda()
        vq, vk, vv = (dev[:, :, i].transpose(1, 2) for i in range(3))
        splat.rotary(rot, vq, vk, Y=vq, Y2=vk)
        torch.cuda.synchronize()
        rotary_check("q in place", vq, qkv[:, :, 0].transpose(1, 2), here, **kw)
        rotary_check("k in place", vk, qkv[:, :, 1].transpose(1, 2), here, **kw)
        assert torch.equal(vv.cpu(), qkv[:, :, 2].transpose(1, 2))


def test_rotary_scaled_and_back(gpu_lib):
    splat = gpu_lib
    kw = dict(factor=8.0, ramp=(1.0, 4.0))
    rot = splat.Rotary(70000, 128, original_len=8192, magnitude=1.25, base=5e5, **kw)
    g = torch.Generator().manual_seed(2)
    x, y = (torch.randn((2, 3, 50, 128), generator=g) for _ in range(2))
    pos = torch.randint(0, 70000, (2, 50), generator=g, dtype=torch.int32)
    fx = splat.rotary(rot, x.cuda(), positions=pos.cuda())
    by = splat.rotary(rot, y.cuda(), positions=pos.cuda(), inverse=True)
    torch.cuda.synchronize()
    rotary_check("scaled", fx, x, pos, R=128, inter=False, magnitude=1.25, base=5e5, original=8192, **kw)
    # the inverse is the transpose: <R x, y> = <x, R' y>, to the sums' fp32 inputs
    lhs, rhs = (fx.double().cpu() * y.double()).sum(), (x.double() * by.double().cpu()).sum()
    assert abs(lhs - rhs) <= 16 * 2.0 ** -24 * (x.double().abs() * by.double().cpu().abs()).sum()


def test_rotary_positions_outside_the_table(gpu_lib):
    splat = gpu_lib
    rot = splat.Rotary(100, 32)
    x = torch.randn((1, 2, 5, 64), device="cuda")
    pos = torch.tensor([[0, 99, 100, -1, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    y = splat.rotary(rot, x, positions=pos)
    torch.cuda.synchronize()
    assert torch.isfinite(y[:, :, :2]).all() and torch.isnan(y[:, :, 2:, :32]).all()
    assert torch.equal(y[..., 32:], x[..., 32:])


def paged(lengths, page, max_pages, heads, d, dtype, seed, spare=3):
    """(k, v) caches of N(0, 1) and a shuffled table, -1 where unused; CPU."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-int(n) // page) for n in lengths]
    order = torch.randperm(sum(need) + spare, generator=g).int()
    table, at = torch.full((len(need), max_pages), -1, dtype=torch.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    k, v = (torch.randn((order.numel(), heads, page, d), generator=g).to(dtype) for _ in range(2))
    return k, v, table


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,R,inter", [(64, 64, False), (128, 32, True), (64, 0, False)])
@pytest.mark.parametrize("page", [1, 16, 128])
@pytest.mark.parametrize("T,starts,counts", [
    (1, [0, 5, 199], None), (1, [7, 0, 16], [1, 0, 1]), (40, [0, 33, 100], [40, 1, 0]), (130, [3, 60, 0], None)])
def test_append(gpu_lib, T, starts, counts, page, d, R, inter, dtype):
    splat = gpu_lib
    print(f"[gpu] append T={T} page={page} d={d} R={R} {dtype}", flush=True)
    B, H, heads = 3, 6, 2
    g = torch.Generator().manual_seed(T + page)
    q, k, v = (torch.randn((B, T, h, d), generator=g).to(dtype).transpose(1, 2) for h in (H, heads, heads))
    n = counts or [T] * B
    kc, vc, table = paged([s + c for s, c in zip(starts, n)], page, -(-260 // page), heads, d, dtype, 1)
    rot = splat.Rotary(400, R, interleaved=inter) if R else None
    dk, dv = kc.cuda(), vc.cuda()
    qr = splat.cache_append(dk, dv, table.cuda(), torch.tensor(starts, dtype=torch.int32).cuda(), k.cuda(),
                            v.cuda(), counts=None if counts is None else
                            torch.tensor(counts, dtype=torch.int32).cuda(), rot=rot, Q=q.cuda())
    torch.cuda.synchronize()
    pos = torch.tensor(starts)[:, None] + torch.arange(T)
    if R:
        k64, km = rotate64(k, pos, R, inter)
        q64, qm = rotate64(q, pos, R, inter)
    else:
        (k64, q64), (km, qm) = (k.double(), q.double()), (torch.zeros_like(x).double() for x in (k, q))
    want_k, want_v, mag = kc.double(), vc.double(), torch.zeros_like(kc).double()
    new = torch.zeros(kc.shape[0], page, dtype=torch.bool)
    for b in range(B):
        q64[b, :, n[b]:] = 0
        for t in range(n[b]):
            p, o = int(table[b, int(pos[b, t]) // page]), int(pos[b, t]) % page
            want_k[p, :, o], want_v[p, :, o], mag[p, :, o] = k64[b, :, t], v[b, :, t].double(), km[b, :, t]
            new[p, o] = True
    assert torch.equal(dv.cpu().double(), want_v)
    got = dk.cpu().double()
    old = ~new[:, None, :, None].expand_as(got)
    assert torch.equal(got[old], kc.double()[old])
    assert ((got - want_k).abs() <= 4 * 2.0 ** -24 * mag + HALF[dtype] * want_k.abs()).all()
    assert ((qr.cpu().double() - q64).abs() <= 4 * 2.0 ** -24 * qm + HALF[dtype] * q64.abs()).all()


def test_append_leaves_out_what_has_no_place(gpu_lib):
    """Bad pages, positions before and past the table: nothing of them is written."""
    splat = gpu_lib
    page, T = 8, 20
    kc = torch.randn((6, 2, page, 64), device="cuda")
    vc = torch.randn_like(kc)
    table = torch.tensor([[0, -1, 3], [6, 1, 2 ** 31 - 1], [4, 5, -7]], dtype=torch.int32, device="cuda")
    start = torch.tensor([-3, 4, 10], dtype=torch.int32, device="cuda")
    k, v = (torch.randn((3, 2, T, 64), device="cuda") for _ in range(2))
    want = [kc.clone(), vc.clone()]
    for b in range(3):
        for t in range(T):
            m = int(start[b]) + t
            p = int(table[b, m // page]) if 0 <= m < 3 * page else -1
            if 0 <= p < 6:
                want[0][p, :, m % page], want[1][p, :, m % page] = k[b, :, t], v[b, :, t]
    splat.cache_append(kc, vc, table, start, k, v)
    torch.cuda.synchronize()
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


MASKS = [("full", {}, 300), ("window", {"w": 20}, 700), ("window_global", {"w": 30, "n_global": 9}, 2500),
         ("strided_local", {"local": 40, "stride": 33}, 1500), ("dilated", {"w": 33, "dilation": 3}, 400),
         ("blocked", {"block": 33}, 300), ("window_rows", {"w": 9, "lo": 40, "hi": 170}, 300), ("none", {}, 50)]


def decode64(Q, kc, vc, table, lengths, M, scale):
    """(O, its bound) in 64 bits."""
    B, H, _, d = Q.shape
    heads, page = kc.shape[1], kc.shape[2]
    O, bound = torch.zeros(Q.shape, dtype=torch.float64), torch.zeros(Q.shape, dtype=torch.float64)
    for b, n in enumerate(lengths):
        cols = torch.from_numpy(np.nonzero(M[n - 1, :n])[0]) if n > 0 else torch.zeros(0, dtype=torch.long)
        if cols.numel() == 0:
            continue
        p, o = table[b].long()[cols // page], cols % page
        k, v = (x[p, :, o].double().transpose(0, 1).repeat_interleave(H // heads, 0) for x in (kc, vc))
        q = Q[b, :, 0].double()
        s = (k @ q[:, :, None])[..., 0] * scale
        a = (k.abs() @ q.abs()[:, :, None])[..., 0] * abs(scale)
        w = torch.softmax(s, -1)
        O[b, :, 0] = (w[:, None] @ v)[:, 0]
        err = w * (C * (2 + a + (w * a).sum(-1, keepdim=True)) + 2.0 ** -16)
        bound[b, :, 0] = (err[:, None] @ v.abs())[:, 0] + HALF[Q.dtype] * O[b, :, 0].abs()
    return O, bound


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,heads", [(2, 2), (6, 2), (40, 1), (64, 16)])
@pytest.mark.parametrize("kind,params,L", MASKS)
def test_decode(gpu_lib, kind, params, L, H, heads, d, dtype):
    splat = gpu_lib
    print(f"[gpu] decode {kind} L={L} H={H},{heads} d={d} {dtype}", flush=True)
    a, M = make(splat, kind, params, L, grad=False)
    g = torch.Generator().manual_seed(L + H)
    for page, lengths in ((16, [L, 1, 0, L // 2, 45 % L]), (128, [L - 1]), (1, [33, 32])):
        max_pages = -(-L // page)
        kc, vc, table = paged(lengths, page, max_pages, heads, d, dtype, L)
        Q = torch.randn((len(lengths), H, 1, d), generator=g).to(dtype)
        for scale in (1 / math.sqrt(d), -0.3):
            O = splat.sparse_mhsa_decode(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(),
                                         torch.tensor(lengths, dtype=torch.int32).cuda(), scale)
            torch.cuda.synchronize()
            want, bound = decode64(Q, kc, vc, table, lengths, M, scale)
            got = O.double().cpu()
            assert torch.isfinite(got).all()
            over = ((got - want).abs() - bound).max().item()
            assert over <= 0, (page, scale, over)


def test_decode_reads_its_row_only(gpu_lib):
    """NaN everywhere but in the row's keys, in unused pages and behind the last
    token: the result does not change."""
    splat = gpu_lib
    for dtype in TYPES:
        a, M = make(splat, "window_global", {"w": 30, "n_global": 9}, 900)
        lengths, page = [700, 899, 3], 16
        kc, vc, table = paged(lengths, page, 57, 2, 64, dtype, 3)
        Q = torch.randn((3, 4, 1, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
        at = torch.tensor(lengths, dtype=torch.int32).cuda()
        clean = splat.sparse_mhsa_decode(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), at, 0.125)
        used = torch.zeros(kc.shape[0], page, dtype=torch.bool)
        for b, n in enumerate(lengths):
            for j in np.nonzero(M[n - 1, :n])[0]:
                used[int(table[b, j // page]), j % page] = True
        hole = ~used[:, None, :, None].expand_as(kc)
        kc[hole], vc[hole] = math.nan, math.inf
        O = splat.sparse_mhsa_decode(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), at, 0.125)
        torch.cuda.synchronize()
        assert torch.equal(O, clean)


def test_decode_bad_lengths_and_pages(gpu_lib):
    """A length outside the mask or the table, a page outside the cache among the
    row's keys: NaN in that sequence alone.  A bad page that the row has no key
    in does not matter."""
    splat = gpu_lib
    L, page = 400, 16
    for H, w in ((2, 5), (2, 399)):         # one split of the keys and several
        a, M = make(splat, "window", {"w": w}, L)
        lengths = [400, 401, -1, 300, 300, 0, 350]
        kc, vc, table = paged([352] * 7, page, 22, 2, 64, torch.float32, 3)
        table[3, 1] = -1           # w = 5: no key of row 299 lies there
        table[4, 299 // page] = 10 ** 6
        Q = torch.randn((7, H, 1, 64))
        O = splat.sparse_mhsa_decode(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(),
                                     torch.tensor(lengths, dtype=torch.int32).cuda(), 0.125)
        torch.cuda.synchronize()
        nan = torch.isnan(O).flatten(1).all(1).tolist()
        fine = torch.isfinite(O).flatten(1).all(1).tolist()
        assert nan == [True, True, True, w != 5, True, False, False]
        assert fine == [not x for x in nan] and (O[5] == 0).all()


def test_scores_of_minus_infinity(gpu_lib):
    """Keys that score -inf weigh nothing; where all do, the result is NaN."""
    splat = gpu_lib
    a, M = make(splat, "full", {}, 300)
    kc, vc, table = paged([300, 300], 16, 19, 1, 64, torch.float32, 3)
    Q = torch.randn((2, 1, 1, 64))
    Q[..., 0] = 1.0
    kc[..., 0] = 0.0
    kc[table[0, :10].long(), :, :, 0] = -math.inf
    kc[table[1, :19].long(), :, :, 0] = -math.inf
    O = splat.sparse_mhsa_decode(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(),
                                 torch.tensor([300, 300], dtype=torch.int32).cuda(), 0.125)
    torch.cuda.synchronize()
    seen = M.copy()
    seen[:, :160] = False
    kc[torch.isinf(kc)] = 0.0
    want, bound = decode64(Q, kc, vc, table, [300, 300], seen, 0.125)
    assert ((O.double().cpu() - want).abs() <= bound)[0].all() and torch.isnan(O[1]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_serving_a_sequence(gpu_lib, dtype):
    """Prefill and then token by token, as a program does it: rotate, append,
    attend.  Every step's row equals the fused forward's over the whole sequence
    (bf16: the forward rounds P and its scaled Q, 2^-8 of the largest values)."""
    splat = gpu_lib
    B, H, d, page, N, T0 = 2, 3, 64, 16, 90, 70
    kind, params = "strided_local", {"local": 24, "stride": 16}
    a, M = make(splat, kind, params, N, grad=False)
    rot = splat.Rotary(N, 32)
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((B, H, N, d), generator=g).to(dtype).cuda() for _ in range(3))
    qr, kr = splat.rotary(rot, q, k)
    whole = splat.sparse_mhsa_fwd(a, qr, kr, v, 0.125)
    kc = torch.full((B * 6, H, page, d), math.nan, dtype=dtype, device="cuda")
    vc = kc.clone()
    table = torch.randperm(B * 6, generator=g).int().reshape(B, 6).cuda()
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    splat.cache_append(kc, vc, table, start, k[:, :, :T0], v[:, :, :T0], rot=rot)
    for m in range(T0, N):
        start.fill_(m)
        step = splat.cache_append(kc, vc, table, start, k[:, :, m:m + 1], v[:, :, m:m + 1], rot=rot,
                                  Q=q[:, :, m:m + 1])
        O = splat.sparse_mhsa_decode(a, step, kc, vc, table, start + 1, 0.125)
        torch.cuda.synchronize()
        assert torch.equal(step, qr[:, :, m:m + 1])
        ref = whole[:, :, m:m + 1].double()
        tol = (8 * HALF[dtype] + 64 * C) * v.double().abs().max()
        assert ((O.double() - ref).abs() <= tol).all(), m


def test_graph_replays_match_eager(gpu_lib):
    """A decode step captured once, replayed as the sequences grow."""
    splat = gpu_lib
    for dtype in TYPES:
        B, H, heads, d, page = 3, 8, 2, 64, 16
        a, _ = make(splat, "window_global", {"w": 300, "n_global": 9}, 700, grad=False)
        assert splat.decode_workspace(a, B, H, heads, d) > 0
        rot = splat.Rotary(700, 64)
        kc, vc, table = (x.cuda() for x in paged([700] * B, page, 44, heads, d, dtype, 3))
        q, k, v = (torch.randn((B, h, 1, d), device="cuda").to(dtype) for h in (H, heads, heads))
        start = torch.tensor([10, 500, 0], dtype=torch.int32, device="cuda")
        length = start + 1
        qr, O = torch.empty_like(q), torch.empty_like(q)
        ws = torch.empty(splat.decode_workspace(a, B, H, heads, d), dtype=torch.uint8, device="cuda")

        def step():
            splat.cache_append(kc, vc, table, start, k, v, rot=rot, Q=q, Qr=qr)
            splat.sparse_mhsa_decode(a, qr, kc, vc, table, length, 0.125, O=O, workspace=ws)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for r in range(4):
            start += 37
            length.copy_(start + 1)
            for x in (q, k, v):
                x.copy_(torch.randn(x.shape, device="cuda"))
            O.zero_(), qr.zero_()
            graph.replay()
            torch.cuda.synchronize()
            ek, ev = kc.clone(), vc.clone()
            eq = splat.cache_append(ek, ev, table, start, k, v, rot=rot, Q=q)
            eO = splat.sparse_mhsa_decode(a, eq, ek, ev, table, length, 0.125)
            torch.cuda.synchronize()
            assert torch.equal(O, eO) and torch.equal(qr, eq) and torch.equal(kc, ek)


def test_refusals(gpu_lib):
    splat = gpu_lib
    rot = splat.Rotary(64, 64)
    x = torch.randn((2, 4, 8, 64), device="cuda")
    bad = [
        lambda: splat.rotary(rot, x[..., ::2]), lambda: splat.rotary(rot, x.half()),
        lambda: splat.rotary(rot, x[0]), lambda: splat.rotary(rot, x[:, :0]),
        lambda: splat.rotary(rot, x, x.bfloat16()), lambda: splat.rotary(rot, x, x[:1]),
        lambda: splat.rotary(rot, x, Y=x[:, :2]), lambda: splat.rotary(rot, x, Y2=x),
        lambda: splat.rotary(rot, x, positions=torch.zeros((2, 8), device="cuda")),
        lambda: splat.rotary(rot, x, positions=torch.zeros((2, 7), dtype=torch.int32, device="cuda")),
        lambda: splat.rotary(rot, torch.randn((1, 1, 1, 32), device="cuda")),
        lambda: splat.rotary(rot, x, Y=x.transpose(1, 2).contiguous().transpose(1, 2)[:, :, :].expand(2, 4, 8, 64)[:, :, :1]),
        # outputs that lie over an input, another output, or themselves
        lambda: splat.rotary(rot, x[:, :2], Y=x[:, 1:3]), lambda: splat.rotary(rot, x, x.clone(), Y=x.clone(), Y2=x),
        lambda: splat.rotary(rot, x, Y=torch.empty((2, 1, 8, 64), device="cuda").expand(2, 4, 8, 64)),
        lambda: splat.rotary(splat.Rotary(64, 128), x),
        lambda: splat.rotary(rot, torch.randn((2, 4, 8, 66), device="cuda")[..., :64]),
    ]
    kc = torch.randn((6, 2, 16, 64), device="cuda")
    vc, table = torch.randn_like(kc), torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    at = torch.zeros(2, dtype=torch.int32, device="cuda")
    k = torch.randn((2, 2, 4, 64), device="cuda")
    app = lambda **kw: splat.cache_append(**{**dict(k_cache=kc, v_cache=vc, table=table, start=at, K=k, V=k), **kw})
    bad += [
        lambda: app(K=x), lambda: app(V=k[:1]), lambda: app(start=at.long()), lambda: app(start=at[:1]),
        lambda: app(table=table[:1]), lambda: app(table=table.long()), lambda: app(counts=at.float()),
        lambda: app(k_cache=kc.bfloat16()), lambda: app(v_cache=kc), lambda: app(v_cache=vc[:3]),
        lambda: app(K=kc[:2, :, :4], V=k), lambda: app(Qr=x), lambda: app(Q=x),
        lambda: app(Q=x[:, :, :4], Qr=k), lambda: app(k_cache=kc[:, :, :12].contiguous(), v_cache=vc[:, :, :12].contiguous()),
        lambda: app(Q=torch.cat((k, k), 1), Qr=kc[:4].view(2, 4, 16, 64)[:, :, :4]),
    ]
    a, _ = make(splat, "window", {"w": 3}, 40, grad=False)
    Q = torch.randn((2, 4, 1, 64), device="cuda")
    dec = lambda **kw: splat.sparse_mhsa_decode(**{**dict(acsr=a, Q=Q, k_cache=kc, v_cache=vc, table=table,
                                                          lengths=at, scale=1.0), **kw})
    big, _ = make(splat, "full", {}, 700, grad=False)
    need = splat.decode_workspace(big, 2, 4, 2, 64)
    assert need > 0
    bad += [
        lambda: dec(Q=x), lambda: dec(Q=Q[:1]), lambda: dec(Q=Q[:, :3].contiguous()), lambda: dec(Q=Q.bfloat16()),
        lambda: dec(lengths=at.long()), lambda: dec(O=Q), lambda: dec(O=Q[:1]), lambda: dec(O=Q.bfloat16()),
        lambda: dec(acsr=big, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda")),
        lambda: dec(acsr=big, workspace=kc.view(-1)), lambda: dec(O=kc.view(-1)[:512].view(2, 4, 1, 64)),
    ]
    # the training calls
    q = torch.randn((1, 2, 40, 64), device="cuda")
    O, lse = splat.sparse_mhsa_fwd_lse(a, q, q, q, 1.0)
    ag, _ = make(splat, "window", {"w": 3}, 40)
    bwd = lambda **kw: splat.sparse_mhsa_bwd(**{**dict(acsr=ag, Q=q, K=q, V=q, O=O, lse=lse, dO=q, scale=1.0), **kw})
    bwd()
    bad += [
        lambda: bwd(acsr=a), lambda: bwd(lse=lse.double()), lambda: bwd(lse=lse[:, :1]), lambda: bwd(dO=q.bfloat16()),
        lambda: bwd(dQ=q), lambda: bwd(dK=O), lambda: bwd(dQ=torch.empty_like(q)[:, :1]),
        lambda: bwd(workspace=torch.empty((2, 1, 2, 39), device="cuda")), lambda: bwd(O=O[:, :, :39]),
        lambda: splat.sparse_mhsa_fwd_lse(a, q, q, q, 1.0, O=q), lambda: splat.sparse_mhsa_fwd_lse(a, q, q, q, 1.0, lse=O),
    ]
    same = torch.empty_like(q)
    bad += [lambda: bwd(dQ=same, dK=same)]
    for i, call in enumerate(bad):
        with pytest.raises((splat.SplatError, TypeError, ValueError)) as e:
            call()
        if isinstance(e.value, splat.SplatError):
            assert e.value.name in ("INVALID_ARG", "UNSUPPORTED"), (i, e.value)
    torch.cuda.synchronize()


@pytest.mark.parametrize("B,T", [(3, 1), (3, 5), (1, 5)])
@pytest.mark.parametrize("order", ["b t h", "b h t"])
def test_joint_projection_in_place(gpu_lib, B, T, order):
    """Q, K and V as views of one buffer, Q and K turned where they are: views that
    take turns share no memory, whatever the batch and the order of axes."""
    splat = gpu_lib
    H, H2, d, page = 4, 2, 64, 16
    rot = splat.Rotary(64, d)
    n = H + 2 * H2

    def views(x):
        x = x if order == "b h t" else x.transpose(1, 2)
        return x[:, :H], x[:, H:H + H2], x[:, H + H2:]

    x = torch.randn((B, n, T, d) if order == "b h t" else (B, T, n, d), device="cuda")
    q, k, v = views(x)
    kc, vc = (torch.zeros((B, H2, page, d), device="cuda") for _ in range(2))
    table = torch.arange(B, dtype=torch.int32, device="cuda")[:, None].contiguous()
    start = torch.arange(B, dtype=torch.int32, device="cuda")
    wq = splat.cache_append(kc, vc, table, start, k, v, rot=rot, Q=q)
    wk, wv = kc.clone(), vc.clone()
    y = x.clone()
    q, k, v = views(y)
    kc.zero_(), vc.zero_()
    splat.cache_append(kc, vc, table, start, k, v, rot=rot, Q=q, Qr=q)
    assert torch.equal(q, wq) and torch.equal(kc, wk) and torch.equal(vc, wv)
    assert torch.equal(k, views(x)[1]) and torch.equal(v, views(x)[2])
    # both turned in place, in one launch
    want = splat.rotary(rot, *views(x)[:2])
    y = x.clone()
    splat.rotary(rot, *views(y)[:2], Y=views(y)[0], Y2=views(y)[1])
    assert torch.equal(views(y)[0], want[0]) and torch.equal(views(y)[1], want[1])
    # shifted by a head they do share memory
    with pytest.raises(splat.SplatError):
        splat.rotary(rot, y[:, :H] if order == "b h t" else y.transpose(1, 2)[:, :H],
                     Y=y[:, 1:H + 1] if order == "b h t" else y.transpose(1, 2)[:, 1:H + 1])


@pytest.mark.parametrize("dtype", TYPES)
def test_decode_of_shared_pages(gpu_lib, dtype):
    """Sequences that share pages (a common beginning), and a page that a table
    names twice."""
    splat = gpu_lib
    a, M = make(splat, "full", {}, 200, grad=False)
    kc, vc, _ = paged([200], 16, 13, 2, 64, dtype, 3, spare=13)
    assert kc.shape[0] == 26
    table = torch.randperm(26, generator=torch.Generator().manual_seed(4)).to(torch.int32).view(2, 13)
    table[1, :7] = table[0, :7]
    table[0, 9] = table[0, 2]
    Q = torch.randn((2, 6, 1, 64), generator=torch.Generator().manual_seed(5)).to(dtype)
    O = splat.sparse_mhsa_decode(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(),
                                 torch.tensor([200, 119], dtype=torch.int32).cuda(), 0.125)
    torch.cuda.synchronize()
    want, bound = decode64(Q, kc, vc, table, [200, 119], M, 0.125)
    assert ((O.double().cpu() - want).abs() <= bound).all()
