"""The attention of a chunk of new tokens over the paged cache, against a plain
64-bit implementation.

Bounds, as for single tokens: C = 32 * 2^-24 of the terms' magnitudes (a score's
error scales its weight, so a weight's are w (2 + A(s) + sum w A(s)) with A(s) the
sum of the score's products' magnitudes), one rounding of O (half a step: 2^-8 in
bf16), and for bf16 one rounding of the weights before they meet V (2^-8; the kernel
of short chunks keeps them as two parts).  The log-sum-exp: C of the mean magnitude
of its scores, its own and 2.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_grad import C, HALF, make as make_mask
from test_gpu_serve import paged

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]

MASKS = [("full", {}, 300), ("window", {"w": 20}, 700), ("window_global", {"w": 30, "n_global": 9}, 1500),
         ("strided_local", {"local": 40, "stride": 33}, 900), ("dilated", {"w": 33, "dilation": 3}, 400),
         ("blocked", {"block": 33}, 300), ("window_rows", {"w": 9, "lo": 40, "hi": 170}, 300), ("none", {}, 50),
         ("causal", {}, 400), ("sliding", {"w": 60, "n_global": 4}, 800), ("strided_local", {"local": 3, "stride": 80}, 1300)]


def make(splat, kind, params, L):
    i, j = np.arange(L)[:, None], np.arange(L)[None, :]
    if kind == "causal":
        return splat.Acsr(splat.Pattern.from_terms(L, [dict(hi_i=1)])), j <= i
    if kind == "sliding":
        w, G = params["w"], params["n_global"]
        pat = splat.Pattern.from_terms(L, [dict(lo_i=1, lo_c=-w, hi_i=1), dict(row_lo=G, hi_c=G - 1)])
        return splat.Acsr(pat), ((j <= i) & (j >= i - w)) | ((j < G) & (i >= G))
    return make_mask(splat, kind, params, L, grad=False)


def chunk64(Q, kc, vc, table, lengths, counts, M, scale, device="cpu"):
    """(O, its bound, lse, its bound) in 64 bits."""
    B, H, T, d = Q.shape
    heads, page = kc.shape[1], kc.shape[2]
    O, bound = (torch.zeros(Q.shape, dtype=torch.float64) for _ in range(2))
    lse = torch.full((B, H, T), -math.inf, dtype=torch.float64)
    lbound = torch.zeros((B, H, T), dtype=torch.float64)
    kc, vc, Q = (x.to(device) for x in (kc, vc, Q))
    for b, (n, c) in enumerate(zip(lengths, counts)):
        if c == 0:
            continue
        m = torch.from_numpy(np.ascontiguousarray(M[n - c:n, :n])).to(device)
        cols = np.arange(n)
        p, o = table[b].long()[cols // page].to(device), torch.from_numpy(cols % page).to(device)
        k, v = (x[p.clamp(min=0), :, o].double().transpose(0, 1).repeat_interleave(H // heads, 0) for x in (kc, vc))
        seen = m.any(0)
        k, v = (torch.where(seen[:, None], x, 0.0) for x in (k, v))
        q = Q[b, :, :c].double()
        s = (q @ k.transpose(1, 2).contiguous() * scale).masked_fill(~m, -math.inf)
        a = q.abs() @ k.abs().transpose(1, 2).contiguous() * abs(scale)
        some = m.any(-1)
        l = torch.logsumexp(s, -1)
        w = torch.softmax(s, -1).masked_fill(~some[:, None], 0.0)
        wa = (w * a).sum(-1, keepdim=True)
        O[b, :, :c] = (w @ v).cpu()
        err = w * (C * (2 + a + wa) + HALF[Q.dtype])
        bound[b, :, :c] = (err @ v.abs()).cpu() + HALF[Q.dtype] * O[b, :, :c].abs()
        lse[b, :, :c] = l.cpu()
        lbound[b, :, :c] = torch.where(some, C * (wa[..., 0] + 2 + l.abs()), 0.0).cpu()
    return O, bound, lse, lbound


def check(got, want):
    O, lse = (x.double().cpu() for x in got)
    over = ((O - want[0]).abs() - want[1]).max().item()
    assert torch.isfinite(O).all() and over <= 0, over
    none = want[2] == -math.inf
    assert torch.equal(lse == -math.inf, none) and (O[none] == 0).all()
    over = ((lse - want[2]).abs() - want[3])[~none]
    assert over.numel() == 0 or over.max().item() <= 0, over.max().item()


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,heads", [(2, 2), (6, 2), (5, 1), (40, 1), (32, 4)])
@pytest.mark.parametrize("kind,params,L", MASKS)
def test_chunk(gpu_lib, kind, params, L, H, heads, d, dtype):
    splat = gpu_lib
    print(f"[gpu] chunk {kind} {params} L={L} H={H},{heads} d={d} {dtype}", flush=True)
    a, M = make(splat, kind, params, L)
    g = torch.Generator().manual_seed(L + H)
    half = L // 2
    for page, T, lengths, counts in ((16, 1, [L, 1, 0, half], [1, 1, 0, 0]), (128, 7, [L, 7, half, 20], [7, 7, 3, 0]),
                                     (1, 33, [L, 40], None), (64, 150, [min(L, 290), half, 1], [min(L, 150), min(half, 131), 1])):
        T = min(T, L)
        n = counts or [T] * len(lengths)
        kc, vc, table = paged(lengths, page, -(-L // page), heads, d, dtype, L)
        Q = torch.randn((len(lengths), H, T, d), generator=g).to(dtype)
        for scale in (1 / math.sqrt(d), -0.3):
            got = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths), scale,
                                          counts=None if counts is None else ints(n))
            torch.cuda.synchronize()
            check(got, chunk64(Q, kc, vc, table, lengths, n, M, scale))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind,params,L,T", [("full", {}, 2500, 3), ("sliding", {"w": 500, "n_global": 64}, 4000, 700),
                                             ("causal", {}, 3000, 1000), ("strided_local", {"local": 100, "stride": 128}, 4000, 40),
                                             ("dilated", {"w": 256, "dilation": 2}, 3000, 300),
                                             ("window_global", {"w": 512, "n_global": 64}, 4096, 513)])
def test_larger(gpu_lib, kind, params, L, T, dtype):
    """Rows over many units and blocks, shared out and not."""
    splat = gpu_lib
    print(f"[gpu] chunk {kind} L={L} T={T} {dtype}", flush=True)
    a, M = make(splat, kind, params, L)
    for d, H, heads, B in ((64, 4, 4, 1), (128, 8, 2, 2)):
        lengths, counts = [L, L - 77][:B], [T, T - T // 3][:B]
        kc, vc, table = paged(lengths, 64, -(-L // 64), heads, d, dtype, L)
        Q = torch.randn((B, H, T, d), generator=torch.Generator().manual_seed(T)).to(dtype)
        got = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths),
                                      1 / math.sqrt(d), counts=ints(counts))
        torch.cuda.synchronize()
        check(got, chunk64(Q, kc, vc, table, lengths, counts, M, 1 / math.sqrt(d), device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1, 5, 60, 200])
def test_reads_its_rows_only(gpu_lib, T, dtype):
    """NaN and infinities in every key that no row of a sequence has, in unused pages,
    behind the last token: the result does not change.  In a key that some rows have:
    only theirs changes."""
    splat = gpu_lib
    a, M = make(splat, "sliding", {"w": 30, "n_global": 9}, 900)
    lengths, counts, page, heads = [700, 899, 260], [T, T, T - T // 2], 16, 2
    kc, vc, table = paged(lengths, page, 57, heads, 64, dtype, 3)
    Q = torch.randn((3, 6, T, 64), generator=torch.Generator().manual_seed(1)).to(dtype)
    run = lambda k, v: splat.sparse_mhsa_chunk(a, Q.cuda(), k.cuda(), v.cuda(), table.cuda(), ints(lengths), 0.125,
                                               counts=ints(counts))
    want = chunk64(Q, kc, vc, table, lengths, counts, M, 0.125)
    check(run(kc, vc), want)
    used = torch.zeros(kc.shape[0], page, dtype=torch.bool)
    for b, (n, c) in enumerate(zip(lengths, counts)):
        for j in np.nonzero(M[n - c:n, :n].any(0))[0]:
            used[int(table[b, j // page]), j % page] = True
    hole = ~used[:, None, :, None].expand_as(kc)
    k, v = kc.clone(), vc.clone()
    k[hole], v[hole] = math.nan, math.inf
    check(run(k, v), want)
    # the newest token's key and value
    for b, n in enumerate(lengths):
        k[int(table[b, (n - 1) // page]), :, (n - 1) % page] = math.nan
        v[int(table[b, (n - 1) // page]), :, (n - 1) % page] = -math.inf
    O, lse = (x.double().cpu() for x in run(k, v))
    for b, c in enumerate(counts):
        assert torch.isnan(O[b, :, c - 1]).all() and torch.isnan(lse[b, :, c - 1]).all()
        assert ((O[b, :, :c - 1] - want[0][b, :, :c - 1]).abs() <= want[1][b, :, :c - 1]).all()
        assert ((lse[b, :, :c - 1] - want[2][b, :, :c - 1]).abs() <= want[3][b, :, :c - 1]).all()
    # an infinite value alone, in a key that has weight
    v = vc.clone()
    v[int(table[0, 699 // page]), :, 699 % page, 5] = math.inf
    O = run(kc, v)[0].double().cpu()[0]
    assert torch.isinf(O[:, counts[0] - 1, 5]).all()
    O[:, counts[0] - 1, 5] = want[0][0, :, counts[0] - 1, 5]
    assert ((O - want[0][0]).abs() <= want[1][0]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [2, 40, 150])
def test_bad_lengths_counts_and_pages(gpu_lib, T, dtype):
    """A length that is none: NaN in the sequence's rows.  A page that is none: NaN in
    the rows that have a key there, in no others.  Counts past T and below 0 are cut."""
    splat = gpu_lib
    L, page = 400, 16
    for w in (5, 399):
        a, M = make(splat, "window", {"w": w}, L)
        lengths = [400, 401, -1, 300, 300, 0, 352, T - 1, 350]
        counts = [T + 5, T, T, T, T, 0, T, T, -3]
        kc, vc, table = paged([352] * 9, page, 22, 2, 64, dtype, 3)
        table[3, 1] = -1
        table[4, (300 - T) // page] = 10 ** 6
        Q = torch.randn((9, 4, T, 64)).to(dtype)
        O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths), 0.125,
                                         counts=ints(counts))
        torch.cuda.synchronize()
        nan = torch.isnan(O).cpu()
        assert torch.equal(torch.isnan(lse).cpu(), nan.all(-1)) and torch.equal(nan.any(-1), nan.all(-1))
        nan = nan.all(-1)
        for b in (0, 1, 2, 7):
            assert nan[b].all()
        assert not nan[5].any() and not nan[6].any() and not nan[8].any()
        assert (O[8] == 0).all() and (lse[8] == -math.inf).all() and (O[5] == 0).all()
        for b, p in ((3, 1), (4, (300 - T) // page)):
            hit = torch.from_numpy(M[300 - T:300, p * page:min((p + 1) * page, 300)].any(1))
            assert torch.equal(nan[b], hit.expand(4, T)), (w, b)
        keep = [6]
        want = chunk64(Q[keep], kc, vc, table[keep], [352], [T], M, 0.125)
        check((O[keep], lse[keep]), want)


def test_scores_of_minus_infinity(gpu_lib):
    """Keys that score -inf weigh nothing; where all do, the result is NaN and the
    log-sum-exp -inf."""
    splat = gpu_lib
    a, M = make(splat, "full", {}, 300)
    for T in (1, 40, 130):
        kc, vc, table = paged([300, 300], 16, 19, 1, 64, torch.float32, 3)
        Q = torch.randn((2, 1, T, 64))
        Q[..., 0] = 1.0
        kc[..., 0] = 0.0
        kc[table[0, :10].long(), :, :, 0] = -math.inf
        kc[table[1, :19].long(), :, :, 0] = -math.inf
        O, lse = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints([300, 300]), 0.125)
        torch.cuda.synchronize()
        seen = M.copy()
        seen[:, :160] = False
        kc[torch.isinf(kc)] = 0.0
        want = chunk64(Q, kc, vc, table, [300, 300], [T, T], seen, 0.125)
        check((O[:1], lse[:1]), [x[:1] for x in want])
        assert torch.isnan(O[1]).all() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_large_scores(gpu_lib, dtype):
    """Scores of hundreds, far apart from tile to tile: the running maximum."""
    splat = gpu_lib
    a, M = make(splat, "causal", {}, 700)
    for T, order in ((6, 1), (6, -1), (200, 1), (200, -1)):
        kc, vc, table = paged([700], 16, 44, 1, 64, dtype, 3)
        ramp = (torch.arange(700) if order > 0 else 699 - torch.arange(700)).float() / 700 * 8
        j = torch.arange(700)
        kc[table[0, j // 16].long(), :, j % 16] += ramp[:, None, None].to(dtype)
        Q = (torch.randn((1, 2, T, 64), generator=torch.Generator().manual_seed(T)) + 1).to(dtype)
        for scale in (0.125, 1.0, -1.0):
            got = splat.sparse_mhsa_chunk(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), ints([700]), scale)
            torch.cuda.synchronize()
            check(got, chunk64(Q, kc, vc, table, [700], [T], M, scale))


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_outputs_and_shared_pages(gpu_lib, dtype):
    splat = gpu_lib
    a, M = make(splat, "causal", {}, 200)
    for T in (3, 90):
        kc, vc, _ = paged([200], 16, 13, 2, 64, dtype, 3, spare=13)
        table = torch.randperm(26, generator=torch.Generator().manual_seed(4)).to(torch.int32).view(2, 13)
        table[1, :7] = table[0, :7]
        table[0, 9] = table[0, 2]
        lengths = [200, 119]
        joint = torch.randn((2, T, 10, 64), generator=torch.Generator().manual_seed(5)).to(dtype)
        Q = joint[:, :, 1:7].transpose(1, 2)
        dev = joint.cuda()
        O = torch.full((2, T, 8, 64), 7.0, dtype=dtype, device="cuda")
        lse = torch.empty((2, 6, T), device="cuda")
        ws = torch.empty(splat.chunk_workspace(a, dtype, 2, 6, 2, T, 64) + 64, dtype=torch.uint8, device="cuda")
        r = splat.sparse_mhsa_chunk(a, dev[:, :, 1:7].transpose(1, 2), kc.cuda(), vc.cuda(), table.cuda(), ints(lengths),
                                    0.125, O=O[:, :, 2:].transpose(1, 2), lse=lse, workspace=ws)
        torch.cuda.synchronize()
        assert r[1].data_ptr() == lse.data_ptr() and (O[:, :, :2] == 7.0).all()
        check((O[:, :, 2:].transpose(1, 2), lse), chunk64(Q, kc, vc, table, lengths, [T, T], M, 0.125))


@pytest.mark.parametrize("dtype", TYPES)
def test_one_token_is_decode(gpu_lib, dtype):
    splat = gpu_lib
    a, M = make(splat, "window_global", {"w": 300, "n_global": 9}, 700)
    kc, vc, table = (x.cuda() for x in paged([700, 333], 16, 44, 2, 128, dtype, 3))
    Q = torch.randn((2, 8, 1, 128), device="cuda").to(dtype)
    O, _ = splat.sparse_mhsa_chunk(a, Q, kc, vc, table, ints([700, 333]), 0.09)
    D = splat.sparse_mhsa_decode(a, Q, kc, vc, table, ints([700, 333]), 0.09)
    assert (O.double() - D.double()).abs().max() <= 2 * (HALF[dtype] + 2.0 ** -12) * vc.double().abs().max()


@pytest.mark.parametrize("dtype", TYPES)
def test_prompts_in_chunks(gpu_lib, dtype):
    """A prompt in ragged chunks and then tokens, as a program does it: rotate,
    append, attend; every row equals the fused forward's over the whole sequence."""
    splat = gpu_lib
    B, H, d, page, N = 2, 3, 64, 16, 230
    a, M = make(splat, "sliding", {"w": 40, "n_global": 4}, N)
    rot = splat.Rotary(N, 32)
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((B, H, N, d), generator=g).to(dtype).cuda() for _ in range(3))
    qr, kr = splat.rotary(rot, q, k)
    whole = splat.sparse_mhsa_fwd(a, qr, kr, v, 0.125)
    kc = torch.full((B * 15, H, page, d), math.nan, dtype=dtype, device="cuda")
    vc = kc.clone()
    table = torch.randperm(B * 15, generator=g).int().reshape(B, 15).cuda()
    tol = (8 * HALF[dtype] + 64 * C) * v.double().abs().max()
    at = [0, 0]
    for T, counts in ((100, [100, 70]), (100, [31, 100]), (1, [1, 1]), (30, [0, 29]), (98, [98, 30])):
        take = lambda x: torch.stack([torch.nn.functional.pad(x[b, :, at[b]:at[b] + counts[b]], (0, 0, 0, T - counts[b]))
                                      for b in range(B)])
        start, n = ints(at), ints(counts)
        step = splat.cache_append(kc, vc, table, start, take(k), take(v), rot=rot, Q=take(q), counts=n)
        O, _ = splat.sparse_mhsa_chunk(a, step, kc, vc, table, start + n, 0.125, counts=n)
        torch.cuda.synchronize()
        for b in range(B):
            ref = whole[b, :, at[b]:at[b] + counts[b]].double()
            assert ((O[b, :, :counts[b]].double() - ref).abs() <= tol).all()
            at[b] += counts[b]
    assert at == [230, 230]


@pytest.mark.parametrize("T", [4, 64])
def test_graph_replays_match_eager(gpu_lib, T):
    splat = gpu_lib
    for dtype in TYPES:
        B, H, heads, d, page = 3, 8, 2, 64, 16
        a, _ = make(splat, "window_global", {"w": 300, "n_global": 9}, 700)
        kc, vc, table = (x.cuda() for x in paged([700] * B, page, 44, heads, d, dtype, 3))
        Q = torch.randn((B, H, T, d), device="cuda").to(dtype)
        length, n = ints([100, 500, T]), ints([T, T, T])
        O, lse = torch.empty_like(Q), torch.empty((B, H, T), device="cuda")
        ws = torch.empty(max(16, splat.chunk_workspace(a, dtype, B, H, heads, T, d)), dtype=torch.uint8, device="cuda")
        step = lambda: splat.sparse_mhsa_chunk(a, Q, kc, vc, table, length, 0.125, counts=n, O=O, lse=lse, workspace=ws)
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
            length += 37
            n.copy_(ints([T, T - r, r]))
            Q.copy_(torch.randn(Q.shape, device="cuda"))
            O.zero_(), lse.zero_()
            graph.replay()
            torch.cuda.synchronize()
            eO, el = splat.sparse_mhsa_chunk(a, Q, kc, vc, table, length, 0.125, counts=n)
            torch.cuda.synchronize()
            assert torch.equal(O, eO) and torch.equal(lse, el)


def test_two_streams_at_once(gpu_lib):
    splat = gpu_lib
    a, _ = make(splat, "causal", {}, 2000)
    kc, vc, table = (x.cuda() for x in paged([2000] * 2, 64, 32, 2, 64, torch.bfloat16, 3))
    Q = [torch.randn((2, 4, 6, 64), device="cuda").bfloat16() for _ in range(2)]
    n = ints([2000, 1700])
    call = lambda q: splat.sparse_mhsa_chunk(a, q, kc, vc, table, n, 0.125)
    want = [call(q) for q in Q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in Q]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        for s, q in zip(streams, Q):
            with torch.cuda.stream(s):
                got.append(call(q))
    torch.cuda.synchronize()
    for k, (O, lse) in enumerate(got):
        assert torch.equal(O, want[k % 2][0]) and torch.equal(lse, want[k % 2][1])


def test_refusals(gpu_lib):
    splat = gpu_lib
    a, _ = make(splat, "window", {"w": 3}, 48)
    kc = torch.randn((6, 2, 16, 64), device="cuda")
    vc, table = torch.randn_like(kc), torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    at = torch.full((2,), 40, dtype=torch.int32, device="cuda")
    Q = torch.randn((2, 4, 8, 64), device="cuda")
    call = lambda **kw: splat.sparse_mhsa_chunk(**{**dict(acsr=a, Q=Q, k_cache=kc, v_cache=vc, table=table, lengths=at,
                                                          scale=1.0), **kw})
    call()
    big, _ = make(splat, "full", {}, 3000)
    need = splat.chunk_workspace(big, torch.float32, 2, 4, 2, 8, 64)
    assert need > 0
    f = lambda *s: torch.empty(s, device="cuda")
    bad = [lambda: call(Q=Q[:1]), lambda: call(Q=Q[:, :3]), lambda: call(Q=Q.bfloat16()), lambda: call(Q=Q.half()),
           lambda: call(Q=Q[..., ::2]), lambda: call(Q=Q[0]), lambda: call(Q=Q[:, :, :0]), lambda: call(Q=Q.cpu()),
           lambda: call(lengths=at.long()), lambda: call(lengths=at[:1]), lambda: call(counts=at.float()),
           lambda: call(counts=at[:1]), lambda: call(O=Q), lambda: call(O=Q[:, :, :4]), lambda: call(O=Q.bfloat16()),
           lambda: call(O=f(2, 4, 1, 64).expand(2, 4, 8, 64)), lambda: call(lse=f(2, 4, 7)),
           lambda: call(lse=f(2, 4, 8).double()), lambda: call(lse=Q.view(-1)[:64].view(2, 4, 8)),
           lambda: call(table=table.long()), lambda: call(table=table[:1]), lambda: call(v_cache=vc[:3]),
           lambda: call(O=kc.view(-1)[:4096].view(2, 4, 8, 64)), lambda: call(k_cache=kc.bfloat16()),
           lambda: call(acsr=big, workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda")),
           lambda: call(acsr=big, workspace=Q.view(-1)) if need <= Q.nbytes else call(Q=Q[:1]),
           lambda: call(acsr=big, workspace=torch.empty(need + 8, dtype=torch.uint8, device="cuda")[8:])]
    for i, g in enumerate(bad):
        with pytest.raises((splat.SplatError, TypeError, ValueError)) as e:
            g()
        if isinstance(e.value, splat.SplatError):
            assert e.value.name in ("INVALID_ARG", "UNSUPPORTED"), (i, e.value)
    torch.cuda.synchronize()
