"""The checked build over the kernels that large launches take: chunks by tiles of 128
rows, weights by blocks of 64 keys, and eviction: no index outside its buffer is recorded,
and every output equals the regular library's bit for bit."""
import ctypes

import pytest
import torch

from test_gpu_checked import _flags, _ptr, _stream, libs  # noqa: F401
from test_gpu_checked_ops import TRAIN
from test_gpu_chunk_tiles import heads_for_tiles

pytestmark = pytest.mark.gpu


def cache_of(kc, vc, table, page):
    return (ctypes.c_int64 * 7)(kc.data_ptr(), vc.data_ptr(), table.data_ptr(), kc.shape[0], kc.shape[1], page, table.shape[1])


@pytest.mark.parametrize("page", [2, 8, 16, 64])
@pytest.mark.parametrize("G,T", [(1, 150), (5, 110)])
@pytest.mark.parametrize("kind,params,L,d", [e for e in TRAIN if e[2] > 100])
def test_large_launches(libs, kind, params, L, d, G, T, page):
    splat, reg, chk = libs
    pattern = splat.Pattern.named(kind, params, L)
    a, B, T = splat.Acsr(pattern), 2, min(T, L)
    heads = heads_for_tiles(splat, a, B, G, T, d)
    H, most = G * heads, -(-L // page)
    weighs = splat.weights_route(a, torch.bfloat16, B, H, heads, T, d, L)[0]
    assert weighs == "tiles" or G == 1
    print(f"[gpu] checked build, tiles {kind} L={L} G={G} heads={heads} T={T} d={d} page={page} {weighs}", flush=True)
    g = torch.Generator("cuda").manual_seed(5)
    kc, vc = (torch.randn((B * most, heads, page, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.randperm(B * most, generator=g, device="cuda").int().view(B, most)
    table[1, :max(0, (L // 2 - T) // page - 1)] = -1            # pages that a window may have left behind
    Q = torch.randn((B, H, T, d), generator=g, device="cuda").bfloat16()
    lengths = torch.tensor([L, max(T, L // 2)], dtype=torch.int32, device="cuda")
    counts = torch.tensor([T, T - T // 3], dtype=torch.int32, device="cuda")
    cache = cache_of(kc, vc, table, page)
    view = lambda x: (ctypes.c_int64 * 5)(x.data_ptr(), x.stride(0), x.stride(1), x.stride(2), x.size(1))
    out = []
    for lib in (reg, chk):
        h = ctypes.c_void_p()
        assert lib.splat_acsr_build(ctypes.byref(pattern.desc), ctypes.byref(h)) == 0
        n = ctypes.c_int64()
        assert lib.splat_chunk_workspace(h, 1, B, H, heads, T, d, ctypes.byref(n)) == 0
        ws, O = torch.empty(max(n.value, 16), dtype=torch.uint8, device="cuda"), torch.empty_like(Q)
        lse, w = torch.empty((B, H, T), device="cuda"), torch.ones((B * most, heads, page), device="cuda")
        _flags(lib) if lib is chk else None
        assert lib.splat_sparse_mhsa_chunk(h, 1, B, T, d, view(Q), cache, _ptr(lengths), _ptr(counts), 0.1, view(O),
                                           _ptr(lse), _ptr(ws), _stream()) == 0, lib.splat_last_error()
        assert lib.splat_cache_weights(h, 1, B, T, d, view(Q), _ptr(lse), cache, _ptr(lengths), _ptr(counts), 0.1, 0.5,
                                       _ptr(w), _ptr(w), _stream()) == 0, lib.splat_last_error()
        torch.cuda.synchronize()
        lib.splat_acsr_destroy(h)
        out.append([x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32) for x in (O, lse, w)])
    assert _flags(chk) == 0
    for x, y in zip(*out):
        assert torch.equal(x, y)


@pytest.mark.parametrize("moves", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("room,budget,first,recent", [(700, 300, 4, 50), (9000, 4097, 64, 512), (20000, 1, 0, 1), (65536, 30000, 0, 0)])
def test_eviction(libs, room, budget, first, recent, dtype, moves):
    splat, reg, chk = libs
    dt, page, heads, d = torch.bfloat16 if dtype == "bf16" else torch.float32, 16, 2, 64
    most, top = -(-room // page), -(-budget // page)
    lengths = torch.tensor([room, budget, budget - 1, room // 2, room + 1, -1], dtype=torch.int32, device="cuda")
    B = len(lengths)
    print(f"[gpu] checked build, eviction room={room} budget={budget} {dtype} moves={moves}", flush=True)
    g = torch.Generator("cuda").manual_seed(5)
    pages = B * (most + top)
    order = torch.randperm(pages, generator=g, device="cuda").int()
    table, to = order[:B * most].view(B, most).clone(), order[B * most:].view(B, top).contiguous()
    table[3, 1] = -1
    k, v = (torch.randn((pages, heads, page, d), generator=g, device="cuda").to(dt) for _ in range(2))
    w = torch.randn((pages, heads, page), generator=g, device="cuda")
    out = []
    for lib in (reg, chk):
        kc, vc, wc = k.clone(), v.clone(), w.clone()
        kept = torch.zeros((B, heads, budget), dtype=torch.int32, device="cuda")
        left = torch.zeros(B, dtype=torch.int32, device="cuda")
        _flags(lib) if lib is chk else None
        assert lib.splat_cache_evict(int(dtype == "bf16"), B, d, cache_of(kc, vc, table, page), _ptr(wc), _ptr(lengths),
                                     budget, first, recent, _ptr(to) if moves else None, top if moves else 0, _ptr(kept),
                                     _ptr(left), _stream()) == 0, lib.splat_last_error()
        torch.cuda.synchronize()
        out.append((kc, vc, wc, kept, left))
    assert _flags(chk) == 0
    for x, y in zip(*out):
        assert torch.equal(x, y)
