"""Training and serving at the largest sizes: sequences of 65536 positions, and
tensors and caches whose byte offsets pass 32 bits.

Bounds as in test_gpu_grad.py, but for sums of up to 65536 terms: one accumulator
adds them in turn and is off by about sqrt(65536) u = 256 u of the terms'
magnitudes, where those tests allow 32 u.
"""
import math

import pytest
import torch

from oracle import masks as om
from test_gpu_grad import HALF
from test_gpu_serve import decode64

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
LONG = 256 * 2.0 ** -24
L = 65536


@pytest.mark.parametrize("d,dtype", [(64, torch.float32), (64, torch.bfloat16), (128, torch.bfloat16)])
def test_training_at_the_longest_sequence(gpu_lib, d, dtype):
    """Window and global tokens, every row and key, against 64 bits, 2048 rows at a
    time."""
    splat = gpu_lib
    w, n_global, scale = 40, 3, 1.0 / math.sqrt(d)
    print(f"[gpu] long training d={d} {dtype}", flush=True)
    a = splat.Acsr(splat.Pattern.window_global(L, w=w, n_global=n_global), grad=True)
    g = torch.Generator(device="cuda").manual_seed(d)
    Q, K, V, dO = (torch.randn((1, 1, L, d), generator=g, device="cuda").to(dtype) for _ in range(4))
    O, lse = splat.sparse_mhsa_fwd_lse(a, Q, K, V, scale)
    dQ, dK, dV = splat.sparse_mhsa_bwd(a, Q, K, V, O, lse, dO, scale)
    torch.cuda.synchronize()

    q, k, v, o, do = (x[0, 0].double() for x in (Q, K, V, O, dO))
    half = HALF[dtype]
    want = {n: torch.zeros_like(q) for n in ("dK", "dV")}
    tol = {n: torch.zeros_like(q) for n in ("dK", "dV")}
    j = torch.arange(L, device="cuda")[None, :]
    for r0 in range(0, L, 2048):
        r = slice(r0, r0 + 2048)
        i = torch.arange(L, device="cuda")[r, None]
        M = ((i - j).abs() <= w) | (i < n_global) | (j < n_global)
        s = (q[r] @ k.T) * scale
        A = (q[r].abs() @ k.abs().T) * scale
        s.masked_fill_(~M, -math.inf)
        l64 = torch.logsumexp(s, -1)
        p = torch.exp(s - l64[:, None])
        ref = p @ v
        pA = (p * A).sum(-1)
        assert ((lse[0, 0, r].double() - l64).abs() <= LONG * (pA + l64.abs() + 1)).all(), r0
        mag = p @ v.abs()
        bound = (LONG * (2 + A) * p) @ v.abs() + (2 * half + LONG * pA[:, None]) * mag + half * ref.abs()
        assert ((o[r] - ref).abs() <= bound).all(), r0
        # the gradients of the lse and O that the call got
        l = lse[0, 0, r].double()[:, None]
        p = torch.exp(s - l)
        ap = p * (2 + A + l.abs())
        dp, adp = do[r] @ v.T, do[r].abs() @ v.abs().T
        delta = (p * dp).sum(-1, keepdim=True)
        off = (do[r] * (o[r] - p @ v)).sum(-1, keepdim=True).abs()
        ds = p * (dp - delta)
        ads = LONG * ap * (adp + (do[r] * o[r]).abs().sum(-1, keepdim=True)) + p * off + half * ds.abs()
        x = scale * (ds @ k)
        assert ((dQ[0, 0, r].double() - x).abs() <= scale * (ads @ k.abs()) + half * x.abs()).all(), r0
        want["dK"] += scale * (ds.T @ q[r])
        tol["dK"] += scale * (ads.T @ q[r].abs())
        want["dV"] += p.T @ do[r]
        tol["dV"] += (LONG * ap + half * p).T @ do[r].abs()
    for n, got in (("dK", dK), ("dV", dV)):
        over = (got[0, 0].double() - want[n]).abs() - tol[n] - half * want[n].abs()
        assert over.max().item() <= 0, n


def test_training_past_four_gigabytes(gpu_lib):
    """530 heads of 65536 rows, 4.4 GB a tensor: the last head equals a launch of
    its own (roundings of bf16 apart)."""
    splat = gpu_lib
    H, d = 530, 64
    a = splat.Acsr(splat.Pattern.window(L, w=5), grad=True)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = [torch.zeros((1, H, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    for t in x:
        t[:, -1].normal_(generator=g)
    O, lse = splat.sparse_mhsa_fwd_lse(a, *x[:3], 0.125)
    got = splat.sparse_mhsa_bwd(a, *x[:3], O, lse, x[3], 0.125)
    one = [t[:, -1:].contiguous() for t in x]
    O1, lse1 = splat.sparse_mhsa_fwd_lse(a, *one[:3], 0.125)
    want = splat.sparse_mhsa_bwd(a, *one[:3], O1, lse1, one[3], 0.125)
    torch.cuda.synchronize()
    for u, v in zip((O, *got), (O1, *want)):
        assert (u[:, -1:] - v).abs().max() <= 2.0 ** -6 * v.abs().max() and v.abs().max() > 0
        assert (u[:, :-1:100] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_cache_past_four_gigabytes(gpu_lib, dtype):
    """Pages at the end of a cache of more than 2^32 bytes: append and decode as in
    a small one, bit for bit."""
    splat = gpu_lib
    d, page, heads, T = 128, 256, 2, 300
    n = 2 ** 32 // (page * heads * d * dtype.itemsize) + 8
    big = [torch.zeros((n, heads, page, d), dtype=dtype, device="cuda") for _ in range(2)]
    small = [torch.zeros((8, heads, page, d), dtype=dtype, device="cuda") for _ in range(2)]
    at = torch.tensor([[1, 4], [7, 2]], dtype=torch.int32, device="cuda")
    start = torch.tensor([3, 200], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    K, V = (torch.randn((2, heads, T, d), generator=g, device="cuda").to(dtype) for _ in range(2))
    Q = torch.randn((2, 8, 1, d), generator=g, device="cuda").to(dtype)
    rot = splat.Rotary(600, d)
    a = splat.Acsr(splat.Pattern.full(600))
    out = []
    for cache, first in ((big, n - 8), (small, 0)):
        table = at + first
        splat.cache_append(*cache, table, start, K, V, rot=rot)
        out.append(splat.sparse_mhsa_decode(a, Q, *cache, table, start + T, 0.1))
    torch.cuda.synchronize()
    assert torch.equal(big[0][-8:], small[0]) and torch.equal(big[1][-8:], small[1])
    assert (big[0][:8] == 0).all() and (big[1][:8] == 0).all()
    assert torch.equal(*out) and out[0].abs().max() > 0


@pytest.mark.parametrize("dtype", TYPES)
def test_decode_at_the_longest_sequence(gpu_lib, dtype):
    splat = gpu_lib
    local, stride, page, d = 3000, 32, 64, 64
    a = splat.Acsr(splat.Pattern.strided_local(L, local, stride))
    lengths = [L, L - 1, 40001]
    g = torch.Generator().manual_seed(3)
    kc, vc = (torch.randn((L // page, 1, page, d), generator=g).to(dtype) for _ in range(2))
    table = torch.randperm(L // page, generator=g).to(torch.int32)[None].repeat(3, 1).contiguous()
    Q = torch.randn((3, 5, 1, d), generator=g).to(dtype)
    O = splat.sparse_mhsa_decode(a, Q.cuda(), kc.cuda(), vc.cuda(), table.cuda(),
                                 torch.tensor(lengths, dtype=torch.int32).cuda(), 0.125)
    torch.cuda.synchronize()

    class Rows:                       # the mask's rows that decode64 asks for
        def __getitem__(self, at):
            i, cut = at
            return om.dense_mask_row("strided_local", {"local": local, "stride": stride}, L, i)[cut]

    want, bound = decode64(Q, kc, vc, table, lengths, Rows(), 0.125)
    assert ((O.double().cpu() - want).abs() <= bound).all()
