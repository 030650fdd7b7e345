"""The backward pass of rows and keys at the mask's edge: keys that no row has,
rows of few keys beside longer ones, values that are not finite at d = 128.

Bounds as in test_gpu_grad.py.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_grad import C, HALF, LARGE, TYPES, backward64, check, inputs, make

pytestmark = pytest.mark.gpu

# masks with whole groups of 128 keys that no row has
NO_ROWS = [("none", {}, 300, 2), ("window_rows", {"w": 40, "lo": 200, "hi": 400}, 1024, 3),
           ("window_rows", {"w": 3, "lo": 900, "hi": 1000}, 1024, 40)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,params,L,heads", NO_ROWS)
def test_groups_of_keys_without_rows(gpu_lib, kind, params, L, heads, d, dtype):
    """dK and dV of keys that no row has are 0, in groups of such keys alone too:
    nothing that a workgroup keeps in LDS reaches them."""
    splat = gpu_lib
    print(f"[gpu] no rows {kind} {params} L={L} heads={heads} d={d} {dtype}", flush=True)
    a, M = make(splat, kind, params, L)
    Q, K, V, dO = inputs(L, d, heads, dtype, L + d)
    dev, scale = [x.cuda() for x in (Q, K, V, dO)], 1.0 / math.sqrt(d)
    O, lse = splat.sparse_mhsa_fwd_lse(a, *dev[:3], scale)
    got = splat.sparse_mhsa_bwd(a, *dev[:3], O, lse, dev[3], scale)
    torch.cuda.synchronize()
    want, bound = backward64(Q, K, V, O.cpu(), lse.cpu(), dO, M, scale)
    for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bound):
        check(name, g, w, b)
    rows, keys = torch.from_numpy(~M.any(1)), torch.from_numpy(~M.any(0))
    assert (got[0].cpu()[:, :, rows] == 0).all()
    assert (got[1].cpu()[:, :, keys] == 0).all() and (got[2].cpu()[:, :, keys] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,params,L,heads", [
    ("dilated", {"w": 3, "dilation": 100}, 300, 2), ("dilated", {"w": 2, "dilation": 130}, 700, 60),
    ("dilated", {"w": 40, "dilation": 16}, 640, 2), ("strided_local", {"local": 7, "stride": 200}, 900, 2)])
def test_large_strides(gpu_lib, kind, params, L, heads, d, dtype):
    splat = gpu_lib
    print(f"[gpu] strides {kind} {params} L={L} heads={heads} d={d} {dtype}", flush=True)
    a, M = make(splat, kind, params, L)
    x, scale = inputs(L, d, heads, dtype, L + d), 1.0 / math.sqrt(d)
    dev = [t.cuda() for t in x]
    O, lse = splat.sparse_mhsa_fwd_lse(a, *dev[:3], scale)
    got = splat.sparse_mhsa_bwd(a, *dev[:3], O, lse, dev[3], scale)
    torch.cuda.synchronize()
    for h in (0, heads - 1):
        one = [t[:, h:h + 1].cpu() for t in (*x[:3], O, lse, x[3])]
        want, bound = backward64(*one, M, scale)
        for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bound):
            check(f"{name} head {h}", g[:, h:h + 1], w, b)


def few(M):
    """Rows whose delta is the sum of p dP itself, not dO.O with the rounded O."""
    n = M.sum(-1)
    return torch.from_numpy((n > 1) & (n <= 32))


# rows of few keys beside longer ones: the first rows of causal masks, rows beside
# global ones, one row alone, groups of one workgroup and of four
BESIDE = [
    ("strided_local", {"local": 128, "stride": 128}, 700, 2), ("strided_local", {"local": 128, "stride": 128}, 700, 130),
    ("strided_local", {"local": 4, "stride": 16}, 900, 3), ("window_global", {"w": 8, "n_global": 8}, 900, 2),
    ("window_global", {"w": 3, "n_global": 2}, 1300, 60), ("window", {"w": 20}, 400, 2),
    ("window_rows", {"w": 40, "lo": 30, "hi": 31}, 300, 2), ("dilated", {"w": 20, "dilation": 3}, 500, 2),
]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,params,L,heads", BESIDE)
def test_rows_of_few_keys_beside_longer_ones(gpu_lib, kind, params, L, heads, d):
    """bf16: the gradients of a row of 2 .. 32 keys do not depend on the rows that
    share its group: dQ of every such row, and dK of the keys that only such rows
    have, without the rounding of O in the bound."""
    splat = gpu_lib
    print(f"[gpu] few keys {kind} {params} L={L} heads={heads} d={d}", flush=True)
    a, M = make(splat, kind, params, L)
    x, scale = inputs(L, d, heads, torch.bfloat16, L + d), 1.0 / math.sqrt(d)
    dev = [t.cuda() for t in x]
    O, lse = splat.sparse_mhsa_fwd_lse(a, *dev[:3], scale)
    got = splat.sparse_mhsa_bwd(a, *dev[:3], O, lse, dev[3], scale)
    torch.cuda.synchronize()
    rows = few(M)
    for h in {0, heads - 1}:
        one = [t[:, h:h + 1].cpu() for t in (*x[:3], O, lse, x[3])]
        want, bound = backward64(*one, M, scale)
        for name, g, w, b in zip(("dQ", "dK", "dV"), got, want, bound):
            check(f"{name} head {h}", g[:, h:h + 1], w, b)
        # the rows without the term: their part of the mask alone, whose rows all have
        # at most 32 keys
        Mf = M & rows.numpy()[:, None]
        want, bound = backward64(*one, Mf, scale)
        keys = torch.from_numpy(Mf.any(0) & ~(M & ~rows.numpy()[:, None]).any(0))
        for k, name, part in ((0, "dQ of rows of few keys", rows), (1, "dK of their keys", keys)):
            if part.any():
                check(f"{name}, head {h}", got[k][:, h:h + 1].cpu()[:, :, part], want[k][:, :, part],
                      bound[k][:, :, part])
    assert rows.any() or kind == "window_rows"


def _not_finite(splat, a, M, T, where, value, x, scale, dtype):
    """Rows and keys that a value in row or key x does not reach are as without it."""
    T[where][:, :, x, 3] = 0.0

    def run():
        O, lse = splat.sparse_mhsa_fwd_lse(a, T["Q"], T["K"], T["V"], scale)
        grads = splat.sparse_mhsa_bwd(a, T["Q"], T["K"], T["V"], O, lse, T["dO"], scale)
        torch.cuda.synchronize()
        return [y.cpu() for y in (O, *grads)]

    clean = run()
    T[where][:, :, x, 3] = value
    got = run()
    rows = M[:, x].copy() if where in ("K", "V") else np.arange(M.shape[0]) == x
    keys = M[rows].any(0)
    rows, keys = torch.from_numpy(~rows), torch.from_numpy(~keys)
    # a row or key that is formed again has its sums in another order: roundings of p,
    # dS, delta and the result, and of fp32's sums
    half = 8 * HALF[dtype] + 256 * C
    for name, g, r, ok in zip(("O", "dQ", "dK", "dV"), got, clean, (rows, rows, keys, keys)):
        g, r = g[:, :, ok].double(), r[:, :, ok].double()
        assert torch.isfinite(g).all(), name
        if g.numel():
            top = r.abs().amax(-1, keepdim=True)
            assert ((g - r).abs() <= half * top + 1e-6).all(), name


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("where", ["K", "V", "Q", "dO"])
@pytest.mark.parametrize("kind,params,L", [
    ("window", {"w": 16}, 300), ("blocked", {"block": 33}, 200), ("dilated", {"w": 9, "dilation": 3}, 250),
    ("strided_local", {"local": 40, "stride": 33}, 200)])
def test_values_that_are_not_finite_in_wide_heads(gpu_lib, kind, params, L, where, value, dtype):
    """d = 128: half tiles and V in LDS, and the rows that are formed again behind them."""
    splat = gpu_lib
    print(f"[gpu] not finite, d=128, {kind} {where} {value} {dtype}", flush=True)
    a, M = make(splat, kind, params, L)
    T = dict(zip(("Q", "K", "V", "dO"), (t.cuda() for t in inputs(L, 128, 2, dtype, 9))))
    _not_finite(splat, a, M, T, where, value, L // 2, 1 / math.sqrt(128), dtype)


@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("where", ["K", "V", "Q", "dO"])
@pytest.mark.parametrize("kind,params,L,heads", [LARGE[0], LARGE[1], LARGE[5]])
def test_large_launches_of_wide_heads_and_values_that_are_not_finite(gpu_lib, kind, params, L, heads,
                                                                    where, value):
    splat = gpu_lib
    a, M = make(splat, kind, params, L)
    T = dict(zip(("Q", "K", "V", "dO"), (t.cuda() for t in inputs(L, 128, heads, torch.bfloat16, 9))))
    _not_finite(splat, a, M, T, where, value, L // 2, 1 / math.sqrt(128), torch.bfloat16)
