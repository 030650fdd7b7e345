"""Training through the masked attention: the forward that keeps the rows'
log-sum-exp and the backward pass, against a plain 64-bit implementation.

Bounds.  u = 2^-24 is fp32's half step and b = 2^-8 bf16's.  A sum of n fp32
terms t is off by about sqrt(n) u sum|t|, at most 16 u sum|t| for the n <= 256
that one accumulator of these sizes adds, so every fp32 quantity below is held to
C = 32 u times the sum of its terms' magnitudes A(.), two stages deep: a score's
error scales its p, so A(p_ij) = p_ij (2 + A(s_ij) + |lse_i|).  With bf16 inputs
p and dS are rounded once for the products that sum them and every output once,
b of its magnitude each.  delta_i = sum_j p_ij dP_ij comes from the O of the
forward, whose error reaches every dS_ij as p_ij |sum_c dO_ic (O - exact O)_ic|:
that term is part of the bound, but for bf16 masks of at most 32 keys a row, where
the call takes it out.
"""
import math

import numpy as np
import pytest
import torch

from oracle import masks as om

pytestmark = pytest.mark.gpu

C = 32 * 2.0 ** -24
HALF = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}

CASES = [
    # kind, params, L, heads: one row, ragged slices and groups, gathered tiles,
    # rows and keys of 33 .. 63, many tiles, columns that every row has
    ("full", {}, 1, 3), ("full", {}, 2, 1), ("full", {}, 33, 2), ("full", {}, 128, 4),
    ("full", {}, 200, 3), ("window", {"w": 0}, 70, 2), ("window", {"w": 5}, 65, 1),
    ("window", {"w": 100}, 321, 2), ("blocked", {"block": 33}, 300, 2),
    ("dilated", {"w": 33, "dilation": 3}, 400, 2), ("dilated", {"w": 8, "dilation": 4}, 7, 2),
    ("strided_local", {"local": 40, "stride": 33}, 500, 2),
    ("strided_local", {"local": 4, "stride": 64}, 600, 2),
    ("window_global", {"w": 3, "n_global": 1}, 1300, 1),
    ("window_global", {"w": 30, "n_global": 70}, 450, 3),
    ("window_rows", {"w": 9, "lo": 40, "hi": 170}, 300, 2),
    ("none", {}, 50, 2),
]
# launches whose groups stay with one workgroup each, and mixed ones: rows of few
# keys, rows and keys of global tokens beside short ones, halves of 32 and less
LARGE = [
    ("window", {"w": 9}, 700, 130), ("window_global", {"w": 70, "n_global": 40}, 900, 60),
    ("strided_local", {"local": 20, "stride": 50}, 1000, 90), ("full", {}, 290, 150),
    ("dilated", {"w": 40, "dilation": 2}, 600, 120), ("window_rows", {"w": 25, "lo": 70, "hi": 400}, 560, 110),
]
TYPES = [torch.float32, torch.bfloat16]


def make(splat, kind, params, L, grad=True):
    if kind == "none":
        return splat.Acsr(splat.Pattern.from_terms(L, []), grad=grad), np.zeros((L, L), dtype=bool)
    if kind == "window_rows":
        w, lo, hi = params["w"], params["lo"], params["hi"]
        pat = splat.Pattern.from_terms(L, [dict(row_lo=lo, row_hi=hi, lo_i=1, lo_c=-w, hi_i=1, hi_c=w)])
        i, j = np.arange(L)[:, None], np.arange(L)[None, :]
        return splat.Acsr(pat, grad=grad), (abs(i - j) <= w) & (i >= lo) & (i < hi)
    return (splat.Acsr(splat.Pattern.named(kind, params, L), grad=grad),
            om.dense_mask(kind, params, L))


def inputs(L, d, heads, dtype, seed, n=4, B=1):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((B, heads, L, d), generator=g).to(dtype) for _ in range(n)]


def forward64(Q, K, V, M, scale):
    """(O, lse, p, A(s)) in 64 bits on the CPU."""
    q, k, v, M = Q.double(), K.double(), V.double(), torch.from_numpy(M)
    s = (q @ k.transpose(-1, -2)) * scale
    a = (q.abs() @ k.abs().transpose(-1, -2)) * abs(scale)
    s = s.masked_fill(~M, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(M.any(-1), lse, 0.0)[..., None])
    return p @ v, lse, p, a


def backward64(Q, K, V, O, lse, dO, M, scale):
    """((dQ, dK, dV), their bounds) of the gradients with the lse given."""
    q, k, v, o, g = (x.double() for x in (Q, K, V, O, dO))
    half, Mt = HALF[Q.dtype], torch.from_numpy(M)
    s = (q @ k.transpose(-1, -2)) * scale
    l = torch.where(Mt.any(-1), lse.double(), 0.0)[..., None]
    p = torch.exp(s - l).masked_fill(~Mt, 0.0)
    ap = p * (2 + (q.abs() @ k.abs().transpose(-1, -2)) * abs(scale) + l.abs())
    dp, adp = g @ v.transpose(-1, -2), g.abs() @ v.abs().transpose(-1, -2)
    delta, adelta = (p * dp).sum(-1, keepdim=True), (g * o).abs().sum(-1, keepdim=True)
    off = (g * (o - p @ v)).sum(-1, keepdim=True).abs()
    if Q.dtype == torch.bfloat16 and M.sum(-1).max() <= 32:
        off = torch.zeros_like(off)
    one = Mt.sum(-1, keepdim=True) == 1
    ds = (p * (dp - delta)).masked_fill(one, 0.0)
    # its error is C of this
    ads = (ap * (adp + adelta) + p * off / C).masked_fill(one, 0.0)
    T = lambda x: x.transpose(-1, -2)
    out = (scale * (ds @ k), scale * (T(ds) @ q), T(p) @ g)
    mag = (abs(scale) * (ads @ k.abs()), abs(scale) * (T(ads) @ q.abs()), T(ap) @ g.abs())
    rnd = (abs(scale) * (ds.abs() @ k.abs()), abs(scale) * (T(ds.abs()) @ q.abs()), T(p) @ g.abs())
    return out, [C * m + half * r + half * x.abs() for x, m, r in zip(out, mag, rnd)]


def check(name, got, want, bound):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), name
    over = ((got - want).abs() - bound).max().item()
    assert over <= 0, f"{name}: {over:.3e} over its bound"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,params,L,heads", CASES)
def test_forward_lse(gpu_lib, kind, params, L, heads, d, dtype):
    splat = gpu_lib
    print(f"[gpu] fwd_lse {kind} {params} L={L} heads={heads} d={d} {dtype}", flush=True)
    Q, K, V = inputs(L, d, heads, dtype, L + d, 3)
    a, M = make(splat, kind, params, L, grad=False)
    for scale in (1.0 / math.sqrt(d), -0.3, 0.0):
        O, lse = splat.sparse_mhsa_fwd_lse(a, Q.cuda(), K.cuda(), V.cuda(), scale)
        torch.cuda.synchronize()
        ref, l64, p, A = forward64(Q, K, V, M, scale)
        assert O.dtype == dtype and lse.dtype == torch.float32
        none = torch.from_numpy(~M.any(-1))
        assert (lse.cpu()[..., none] == -math.inf).all() and (O.cpu()[..., none, :] == 0).all()
        err = (lse.double().cpu() - l64)[..., ~none]
        worst = ((p * A).sum(-1) + l64.abs() + 1)[..., ~none] * C
        assert (err.abs() <= worst).all(), scale
        half = HALF[dtype]
        # p rounded in the numerator and in the sum it is divided by
        bound = (C * (2 + A) * p) @ V.double().abs() + 2 * half * (p @ V.double().abs()) + half * ref.abs()
        bound += C * (p * A).sum(-1, keepdim=True) * (p @ V.double().abs())
        check("O", O, ref, bound)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,params,L,heads", CASES)
def test_backward(gpu_lib, kind, params, L, heads, d, dtype):
    splat = gpu_lib
    print(f"[gpu] bwd {kind} {params} L={L} heads={heads} d={d} {dtype}", flush=True)
    Q, K, V, dO = inputs(L, d, heads, dtype, 2 * L + d)
    a, M = make(splat, kind, params, L)
    dev = [x.cuda() for x in (Q, K, V, dO)]
    for scale in (1.0 / math.sqrt(d), -0.3, 0.0):
        O, lse = splat.sparse_mhsa_fwd_lse(a, *dev[:3], scale)
        got = splat.sparse_mhsa_bwd(a, *dev[:3], O, lse, dev[3], scale)
        torch.cuda.synchronize()
        want, bound = backward64(Q, K, V, O.cpu(), lse.cpu(), dO, M, scale)
        for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bound):
            assert g.dtype == dtype
            check(f"{name} scale {scale}", g, w, b)
        again = splat.sparse_mhsa_bwd(a, *dev[:3], O, lse, dev[3], scale)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, again))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,params,L,heads", LARGE)
def test_backward_of_large_launches(gpu_lib, kind, params, L, heads, d):
    """bf16: the first and the last heads of launches that fill the chip."""
    splat = gpu_lib
    print(f"[gpu] bwd large {kind} {params} L={L} heads={heads} d={d}", flush=True)
    x = inputs(L, d, heads, torch.bfloat16, L + heads)
    a, M = make(splat, kind, params, L)
    dev, scale = [t.cuda() for t in x], 1.0 / math.sqrt(d)
    O, lse = splat.sparse_mhsa_fwd_lse(a, *dev[:3], scale)
    got = splat.sparse_mhsa_bwd(a, *dev[:3], O, lse, dev[3], scale)
    torch.cuda.synchronize()
    for h in (0, heads - 1):
        one = [t[:, h:h + 1].cpu() for t in (*x[:3], O, lse, x[3])]
        want, bound = backward64(*one, M, scale)
        for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bound):
            check(f"{name} head {h}", g[:, h:h + 1], w, b)


@pytest.mark.parametrize("where", ["K", "V", "Q", "dO"])
@pytest.mark.parametrize("kind,params,L,heads", [LARGE[0], LARGE[1], LARGE[5]])
def test_large_launches_and_values_that_are_not_finite(gpu_lib, kind, params, L, heads, where):
    """As above, where one workgroup has a group: a row or key with NaN."""
    splat = gpu_lib
    d, scale, x = 64, 0.125, L // 2
    a, M = make(splat, kind, params, L)
    T = dict(zip(("Q", "K", "V", "dO"), (t.cuda() for t in inputs(L, d, heads, torch.bfloat16, 9))))
    T[where][:, :, x, 3] = 0.0

    def run():
        O, lse = splat.sparse_mhsa_fwd_lse(a, T["Q"], T["K"], T["V"], scale)
        grads = splat.sparse_mhsa_bwd(a, T["Q"], T["K"], T["V"], O, lse, T["dO"], scale)
        torch.cuda.synchronize()
        return [y.cpu() for y in (O, *grads)]

    clean = run()
    T[where][:, :, x, 3] = math.nan
    got = run()
    rows = M[:, x].copy() if where in ("K", "V") else np.arange(L) == x
    keys = M[rows].any(0)
    rows, keys = torch.from_numpy(~rows), torch.from_numpy(~keys)
    for g, r, ok in zip(got, clean, (rows, rows, keys, keys)):
        g, r = g[:, :, ok].double(), r[:, :, ok].double()
        assert torch.isfinite(g).all()
        if g.numel():
            top = r.abs().amax(-1, keepdim=True)
            assert ((g - r).abs() <= 8 * HALF[torch.bfloat16] * top + 1e-6).all()


@pytest.mark.parametrize("kind,params,L", [("window", {"w": 6}, 40), ("strided_local", {"local": 5, "stride": 7}, 45)])
def test_gradients_are_the_differences(gpu_lib, kind, params, L):
    """fp32: each gradient along a direction against the change of sum(O dO),
    taken in 64 bits at +-h: third-order terms of size h^2."""
    splat = gpu_lib
    d, scale, h = 64, 0.125, 1e-4
    Q, K, V, dO = inputs(L, d, 2, torch.float32, 5)
    a, M = make(splat, kind, params, L)
    dev = [x.cuda() for x in (Q, K, V, dO)]
    O, lse = splat.sparse_mhsa_fwd_lse(a, *dev[:3], scale)
    got = splat.sparse_mhsa_bwd(a, *dev[:3], O, lse, dev[3], scale)
    torch.cuda.synchronize()
    g = torch.Generator().manual_seed(1)
    for k in range(3):
        way = torch.randn(Q.shape, generator=g).double()
        f = []
        for sign in (1, -1):
            x = [Q.double(), K.double(), V.double()]
            x[k] = x[k] + sign * h * way
            f.append((forward64(*x, M, scale)[0] * dO.double()).sum().item())
        slope, mine = (f[0] - f[1]) / (2 * h), (got[k].double().cpu() * way).sum().item()
        size = (got[k].double().cpu().abs() * way.abs()).sum().item()
        assert abs(slope - mine) <= 1e-5 * size


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("where", ["K", "V", "Q", "dO"])
@pytest.mark.parametrize("kind,params,L", [("window", {"w": 16}, 300), ("blocked", {"block": 33}, 200),
                                           ("dilated", {"w": 9, "dilation": 3}, 250),
                                           ("strided_local", {"local": 40, "stride": 33}, 200)])
def test_a_value_that_is_not_finite_stays_with_its_keys(gpu_lib, kind, params, L, where, value, dtype):
    """Row or key x holds an infinity or a NaN.  The rows without it (and the
    gradients that only they reach) are as without it."""
    splat = gpu_lib
    d, scale, x = 64, 0.125, L // 2
    print(f"[gpu] not finite {kind} {where} {value} {dtype}", flush=True)
    a, M = make(splat, kind, params, L)
    T = dict(zip(("Q", "K", "V", "dO"), inputs(L, d, 2, dtype, 9)))

    def run(t):
        dev = {k: v.cuda() for k, v in t.items()}
        O, lse = splat.sparse_mhsa_fwd_lse(a, dev["Q"], dev["K"], dev["V"], scale)
        grads = splat.sparse_mhsa_bwd(a, dev["Q"], dev["K"], dev["V"], O, lse, dev["dO"], scale)
        torch.cuda.synchronize()
        return [y.cpu() for y in (O, lse, *grads)]

    T[where][:, :, x, 3] = 0.0
    clean = run(T)
    T[where][:, :, x, 3] = value
    O, lse, dQ, dK, dV = run(T)
    # rows whose scores, O or dP the value reaches; keys that those rows have
    rows = M[:, x].copy() if where in ("K", "V") else np.arange(L) == x
    keys = M[rows].any(0)
    rows, keys = torch.from_numpy(~rows), torch.from_numpy(~keys)
    half = 2 * HALF[dtype] + 64 * C   # the sums' order differs where a row is formed again
    for name, got, ref, ok in (("O", O, clean[0], rows), ("dQ", dQ, clean[2], rows),
                               ("dK", dK, clean[3], keys), ("dV", dV, clean[4], keys)):
        g, r = got[:, :, ok].double(), ref[:, :, ok].double()
        assert torch.isfinite(g).all(), name
        top = r.abs().amax(-1, keepdim=True)
        assert ((g - r).abs() <= half * 4 * top + 1e-6).all(), name
    if where != "dO":
        assert torch.isfinite(lse[:, :, rows]).all()


def test_a_row_with_one_key_has_no_gradient_of_its_scores(gpu_lib):
    splat = gpu_lib
    for dtype in TYPES:
        for d in (64, 128):
            M = np.zeros((90, 90), dtype=np.uint8)
            M[:, 7] = 1
            M[40:, 7] = 0
            M[40:, 60] = 1
            a = splat.Acsr(mask=M, grad=True)
            Q, K, V, dO = (x.cuda() for x in inputs(90, d, 2, dtype, 3))
            O, lse = splat.sparse_mhsa_fwd_lse(a, Q, K, V, 0.7)
            dQ, dK, dV = splat.sparse_mhsa_bwd(a, Q, K, V, O, lse, dO, 0.7)
            torch.cuda.synchronize()
            assert (dQ == 0).all() and (dK == 0).all()
            want, bound = backward64(*(x.cpu() for x in (Q, K, V, O, lse, dO)), M.astype(bool), 0.7)
            check("dV", dV, want[2], bound[2])


def test_large_scores(gpu_lib):
    """Scores of hundreds: p stays a probability, nothing overflows."""
    splat = gpu_lib
    for dtype in TYPES:
        Q, K, V, dO = inputs(150, 64, 2, dtype, 8)
        Q = Q * 30
        a, M = make(splat, "window", {"w": 20}, 150)
        dev = [x.cuda() for x in (Q, K, V, dO)]
        O, lse = splat.sparse_mhsa_fwd_lse(a, *dev[:3], 0.125)
        got = splat.sparse_mhsa_bwd(a, *dev[:3], O, lse, dev[3], 0.125)
        torch.cuda.synchronize()
        want, bound = backward64(Q, K, V, O.cpu(), lse.cpu(), dO, M, 0.125)
        for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bound):
            check(name, g, w, b)


def test_scores_of_minus_infinity(gpu_lib):
    """A row whose keys all score -inf gets NaN (both types); the others are as if
    they were not there."""
    splat = gpu_lib
    for dtype in TYPES:
        Q, K, V = inputs(200, 64, 2, dtype, 3, 3)
        a, M = make(splat, "window", {"w": 10}, 200, grad=False)
        Q[..., 0], K[..., 0] = 1.0, 0.0
        K[:, :, :60, 0] = -math.inf
        O, lse = splat.sparse_mhsa_fwd_lse(a, Q.cuda(), K.cuda(), V.cuda(), 0.125)
        torch.cuda.synchronize()
        assert torch.isnan(O[:, :, :50]).all() and (lse[:, :, :50] == -math.inf).all()
        assert torch.isfinite(O[:, :, 50:]).all() and torch.isfinite(lse[:, :, 50:]).all()


def test_batches_match_single_heads(gpu_lib):
    """A (batch, head) on its own gives what it gives among others."""
    splat = gpu_lib
    for dtype in TYPES:
        a, _ = make(splat, "window_global", {"w": 30, "n_global": 5}, 333)
        x = [t.cuda() for t in inputs(333, 64, 3, dtype, 4, B=2)]
        O, lse = splat.sparse_mhsa_fwd_lse(a, *x[:3], 0.125)
        got = splat.sparse_mhsa_bwd(a, *x[:3], O, lse, x[3], 0.125)
        one = [t[1:, 2:].clone() for t in (*x[:3], O, lse, x[3])]
        alone = splat.sparse_mhsa_bwd(a, *one, 0.125)
        torch.cuda.synchronize()
        for g, s in zip(got, alone):
            ref = g[1:, 2:].double()
            assert ((s.double() - ref).abs() <= (HALF[dtype] * 2 + 64 * C) * ref.abs().amax() ).all()


def test_graph_replays_match_eager(gpu_lib):
    splat = gpu_lib
    for dtype in TYPES:
        a, _ = make(splat, "window_global", {"w": 40, "n_global": 8}, 500)
        sets = [[t.cuda() for t in inputs(500, 64, 4, dtype, s)] for s in range(4)]
        Q, K, V, dO = (t.clone() for t in sets[0])
        O, dQ, dK, dV = (torch.empty_like(Q) for _ in range(4))
        lse = torch.empty(Q.shape[:3], device="cuda")
        ws = torch.empty((2, *Q.shape[:3]), device="cuda")

        def step():
            splat.sparse_mhsa_fwd_lse(a, Q, K, V, 0.125, O=O, lse=lse)
            splat.sparse_mhsa_bwd(a, Q, K, V, O, lse, dO, 0.125, dQ=dQ, dK=dK, dV=dV, workspace=ws)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        for r in (1, 2, 3, 0):
            for x, y in zip((Q, K, V, dO), sets[r]):
                x.copy_(y)
            for x in (O, lse, dQ, dK, dV, ws):
                x.zero_()
            graph.replay()
            torch.cuda.synchronize()
            eO, el = splat.sparse_mhsa_fwd_lse(a, *sets[r][:3], 0.125)
            eager = (eO, el, *splat.sparse_mhsa_bwd(a, *sets[r][:3], eO, el, sets[r][3], 0.125))
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip((O, lse, dQ, dK, dV), eager)), r


@pytest.mark.parametrize("dtype", TYPES)
def test_autograd(gpu_lib, dtype):
    """A layer's attention from its projections' layout: rotation, attention, and
    the gradients of everything, against 64-bit autograd."""
    from paper_2407_16847_amd import autograd as sag
    from test_host_serve import frequencies
    splat = gpu_lib
    B, H, L, d, R, scale = 2, 3, 150, 64, 32, 0.125
    a, M = make(splat, "window_global", {"w": 40, "n_global": 5}, L)
    rot = splat.Rotary(L, R)
    g = torch.Generator().manual_seed(3)
    x = [torch.randn((B, L, H, d), generator=g).to(dtype) for _ in range(3)]
    dO = torch.randn((B, H, L, d), generator=g).to(dtype)
    leaf = [t.cuda().requires_grad_() for t in x]
    q, k, v = (t.transpose(1, 2) for t in leaf)
    O = sag.sparse_mhsa(a, sag.rotary(rot, q), sag.rotary(rot, k), v.contiguous(), scale)
    O.backward(dO.cuda())
    torch.cuda.synchronize()

    ref = [t.double().requires_grad_() for t in x]
    ang = torch.arange(L).double()[:, None] * torch.from_numpy(frequencies(R))

    def turn(t):
        u, w = t[..., :R // 2], t[..., R // 2:R]
        c, s = ang.cos(), ang.sin()
        return torch.cat((u * c - w * s, w * c + u * s, t[..., R:]), -1)

    rq, rk, rv = (t.transpose(1, 2) for t in ref)
    s = (turn(rq) @ turn(rk).transpose(-1, -2) * scale).masked_fill(~torch.from_numpy(M), -math.inf)
    out = torch.softmax(s, -1) @ rv
    out.backward(dO.double())
    # roundings of the rotated inputs, O, p, dS and the results, each 2^-8 of values
    # up to the largest; fp32: C of them, n <= 150 terms deep
    for name, got, want in [("O", O, out)] + list(zip(("dQ", "dK", "dV"), [t.grad for t in leaf],
                                                     [t.grad for t in ref])):
        assert got.dtype == dtype
        tol = (6 * HALF[dtype] + 8 * C) * want.abs().max().item()
        assert (got.detach().double().cpu() - want.detach()).abs().max().item() <= tol, name

    with torch.no_grad():
        assert torch.equal(sag.sparse_mhsa(a, q.contiguous(), k.contiguous(), v.contiguous(), scale),
                           splat.sparse_mhsa_fwd(a, q.contiguous(), k.contiguous(), v.contiguous(), scale))
    b, _ = make(splat, "window", {"w": 4}, L, grad=False)
    with pytest.raises(ValueError, match="grad=True"):
        sag.sparse_mhsa(b, q.contiguous(), k.contiguous(), v.contiguous(), scale)


def test_another_stream(gpu_lib):
    """Everything runs on the current stream: work queued behind a long kernel on
    a side stream, and read there."""
    splat = gpu_lib
    a, M = make(splat, "window", {"w": 30}, 400)
    Q, K, V, dO = inputs(400, 64, 4, torch.bfloat16, 3)
    side = torch.cuda.Stream()
    dev = [torch.zeros(x.shape, dtype=x.dtype, device="cuda") for x in (Q, K, V, dO)]
    host = [x.cuda() for x in (Q, K, V, dO)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        for x, y in zip(dev, host):
            x.copy_(y)
        O, lse = splat.sparse_mhsa_fwd_lse(a, *dev[:3], 0.125)
        got = splat.sparse_mhsa_bwd(a, *dev[:3], O, lse, dev[3], 0.125)
    side.synchronize()
    eO, el = splat.sparse_mhsa_fwd_lse(a, *host[:3], 0.125)
    eager = splat.sparse_mhsa_bwd(a, *host[:3], eO, el, host[3], 0.125)
    torch.cuda.synchronize()
    assert torch.equal(O, eO) and all(torch.equal(x, y) for x, y in zip(got, eager))


def test_two_streams_at_once(gpu_lib):
    """One handle's calls on two streams, neither waiting for the other: the
    workspaces are the calls' own."""
    splat = gpu_lib
    a, M = make(splat, "window_global", {"w": 60, "n_global": 20}, 1500)
    sides = [torch.cuda.Stream() for _ in range(2)]
    x = [[t.cuda() for t in inputs(1500, 64, 6, torch.bfloat16, 7 + k)] for k in range(2)]

    def step(q, k, v, do):
        O, lse = splat.sparse_mhsa_fwd_lse(a, q, k, v, 0.125)
        return (O, *splat.sparse_mhsa_bwd(a, q, k, v, O, lse, do, 0.125))

    want = [step(*t) for t in x]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for k, side in enumerate(sides):
            with torch.cuda.stream(side):
                got[k].append(step(*x[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for r in got[k]:
            assert all(torch.equal(u, v) for u, v in zip(r, want[k]))
