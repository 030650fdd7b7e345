"""The chunk's calls in the checked build: no index outside its buffer is recorded,
and every output equals the regular library's bit for bit."""
import ctypes

import pytest
import torch

from test_gpu_checked import _flags, _ptr, _stream, libs  # noqa: F401
from test_gpu_checked_ops import TRAIN

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [2, 90])
@pytest.mark.parametrize("kind,params,L,d", [e for e in TRAIN if e[2] > 100])
def test_no_out_of_range_index(libs, kind, params, L, d, T, dtype):
    splat, reg, chk = libs
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    page, B, H, heads = 8, 3, 4, 2
    most = -(-L // page)
    g = torch.Generator("cuda").manual_seed(5)
    kc, vc = (torch.randn((B * most, heads, page, d), generator=g, device="cuda").to(dt) for _ in range(2))
    table = torch.randperm(B * most, generator=g, device="cuda").int().view(B, most)
    Q = torch.randn((B, H, T, d), generator=g, device="cuda").to(dt)
    lengths = torch.tensor([L, T, L // 2], dtype=torch.int32, device="cuda")
    counts = torch.tensor([T, T, min(T, L // 2) - 1], dtype=torch.int32, device="cuda")
    cache = (ctypes.c_int64 * 7)(kc.data_ptr(), vc.data_ptr(), table.data_ptr(), B * most, heads, page, most)
    view = lambda x: (ctypes.c_int64 * 5)(x.data_ptr(), x.stride(0), x.stride(1), x.stride(2), x.size(1))
    print(f"[gpu] checked build, chunk {kind} {params} L={L} T={T} d={d} {dtype}", flush=True)
    out = []
    for lib in (reg, chk):
        h = ctypes.c_void_p()
        assert lib.splat_acsr_build(ctypes.byref(splat.Pattern.named(kind, params, L).desc), ctypes.byref(h)) == 0
        n = ctypes.c_int64()
        code = int(dtype == "bf16")
        assert lib.splat_chunk_workspace(h, code, B, H, heads, T, d, ctypes.byref(n)) == 0
        ws, O = torch.empty(max(n.value, 16), dtype=torch.uint8, device="cuda"), torch.empty_like(Q)
        lse, w = torch.empty((B, H, T), device="cuda"), torch.ones((B * most, heads, page), device="cuda")
        _flags(lib) if lib is chk else None
        assert lib.splat_sparse_mhsa_chunk(h, code, B, T, d, view(Q), cache, _ptr(lengths), _ptr(counts), 0.1, view(O),
                                           _ptr(lse), _ptr(ws), _stream()) == 0, lib.splat_last_error()
        assert lib.splat_cache_weights(h, code, B, T, d, view(Q), _ptr(lse), cache, _ptr(lengths), _ptr(counts), 0.1, 0.5,
                                       _ptr(w), _ptr(w), _stream()) == 0, lib.splat_last_error()
        torch.cuda.synchronize()
        lib.splat_acsr_destroy(h)
        out.append((O, lse, w))
    assert _flags(chk) == 0
    for x, y in zip(*out):
        assert torch.equal(x, y)
