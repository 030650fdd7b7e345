"""The training and serving calls in the checked build: no index outside its
buffer is recorded, and every output equals the regular library's bit for bit."""
import ctypes

import pytest
import torch

import workloads
from test_gpu_checked import EDGE, _flags, _ptr, _stream, libs  # noqa: F401

pytestmark = pytest.mark.gpu


def _train(splat, lib, pattern, w, Q, K, V, dO):
    """The training calls once; {name: output tensor}."""
    h = ctypes.c_void_p()
    assert lib.splat_acsr_build_ex(ctypes.byref(pattern.desc), splat.PLAN_GRAD, ctypes.byref(h)) == 0
    dt, st = (1 if w.dtype == "bf16" else 0), _stream()
    out = {n: torch.empty_like(Q) for n in ("O", "dQ", "dK", "dV")}
    out["lse"] = torch.empty(Q.shape[:3], dtype=torch.float32, device="cuda")
    ws = torch.empty((2, *Q.shape[:3]), dtype=torch.float32, device="cuda")
    try:
        assert lib.splat_sparse_mhsa_fwd_lse(h, dt, w.B, w.H, w.d, _ptr(Q), _ptr(K), _ptr(V), w.scale,
                                             _ptr(out["O"]), _ptr(out["lse"]), st) == 0
        assert lib.splat_sparse_mhsa_bwd(h, dt, w.B, w.H, w.d, _ptr(Q), _ptr(K), _ptr(V),
                                         _ptr(out["O"]), _ptr(out["lse"]), _ptr(dO), w.scale,
                                         _ptr(out["dQ"]), _ptr(out["dK"]), _ptr(out["dV"]), _ptr(ws),
                                         st) == 0, lib.splat_last_error()
        torch.cuda.synchronize()
    finally:
        lib.splat_acsr_destroy(h)
    return out


TRAIN = EDGE + [("window_global", {"w": 70, "n_global": 40}, 900, 64), ("full", {}, 290, 128),
                ("strided_local", {"local": 20, "stride": 50}, 1000, 128)]


@pytest.mark.parametrize("heads", [2, 60])
@pytest.mark.parametrize("kind,params,L,d", TRAIN)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_has_no_out_of_range_index(libs, kind, params, L, d, dtype, heads):
    splat, reg, chk = libs
    w = workloads.Workload("train", 1, heads, L, d, dtype, workloads.make_pattern(kind, **params), 1.0, 7)
    print(f"[gpu] checked build, training {kind} {params} L={L} d={d} {dtype} heads={heads}", flush=True)
    Q, K, V = (x.cuda() for x in workloads.make_qkv(w))
    dO = torch.randn(Q.shape, generator=torch.Generator("cuda").manual_seed(1), device="cuda").to(Q.dtype)
    pat = splat.Pattern.named(kind, params, L)
    assert _flags(chk) >= 0
    ref, got = (_train(splat, lib, pat, w, Q, K, V, dO) for lib in (reg, chk))
    assert _flags(chk) == 0
    for name in ref:
        assert torch.equal(ref[name], got[name]), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind,params,L,d", [e for e in TRAIN if e[2] > 1])
def test_decode_has_no_out_of_range_index(libs, kind, params, L, d, dtype):
    splat, reg, chk = libs
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    page, B, H, heads = 8, 3, 4, 2
    most = -(-L // page)
    g = torch.Generator("cuda").manual_seed(5)
    kc, vc = (torch.randn((B * most, heads, page, d), generator=g, device="cuda").to(dt) for _ in range(2))
    table = torch.randperm(B * most, generator=g, device="cuda").int().view(B, most)
    Q = torch.randn((B, H, 1, d), generator=g, device="cuda").to(dt)
    lengths = torch.tensor([L, 1, L // 2], dtype=torch.int32, device="cuda")
    cache = (ctypes.c_int64 * 7)(kc.data_ptr(), vc.data_ptr(), table.data_ptr(), B * most, heads, page, most)
    print(f"[gpu] checked build, decode {kind} {params} L={L} d={d} {dtype}", flush=True)
    out = []
    for lib in (reg, chk):
        h = ctypes.c_void_p()
        assert lib.splat_acsr_build(ctypes.byref(splat.Pattern.named(kind, params, L).desc), ctypes.byref(h)) == 0
        n = ctypes.c_int64()
        assert lib.splat_decode_workspace(h, B, H, heads, d, ctypes.byref(n)) == 0
        ws, O = torch.empty(max(n.value, 16), dtype=torch.uint8, device="cuda"), torch.empty_like(Q)
        _flags(lib) if lib is chk else None
        assert lib.splat_sparse_mhsa_decode(h, int(dtype == "bf16"), B, H, d, _ptr(Q), cache, _ptr(lengths),
                                            0.1, _ptr(O), _ptr(ws), _stream()) == 0, lib.splat_last_error()
        torch.cuda.synchronize()
        lib.splat_acsr_destroy(h)
        out.append(O)
    assert _flags(chk) == 0 and torch.equal(*out)
