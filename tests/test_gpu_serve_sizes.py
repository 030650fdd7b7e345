"""Rotation and append of many sequences and of many heads: limits are those of
B * T and of the heads, not of their product."""
import pytest
import torch

from test_gpu_serve import TYPES, rotary_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("B,H,T,d", [(4096, 32, 1, 64), (70001, 1, 1, 64), (1, 70001, 1, 64),
                                     (2, 140000, 1, 64), (3, 1, 25000, 128)])
def test_rotation_of_packed_tokens(gpu_lib, B, H, T, d, dtype):
    splat = gpu_lib
    print(f"[gpu] packed B={B} H={H} T={T} d={d} {dtype}", flush=True)
    g = torch.Generator().manual_seed(B + H)
    rot = splat.Rotary(30000, 32)
    x = torch.randn((B, H, T, d), generator=g).to(dtype)
    pos = torch.randint(0, 30000, (B, T), generator=g, dtype=torch.int32)
    y = splat.rotary(rot, x.cuda(), positions=pos.cuda())
    q, k = splat.rotary(rot, x.cuda(), x.cuda(), positions=pos.cuda())
    torch.cuda.synchronize()
    rotary_check("y", y, x, pos, R=32, inter=False)
    assert torch.equal(q, y) and torch.equal(k, y)


@pytest.mark.parametrize("dtype", TYPES)
def test_append_of_a_token_to_many_sequences(gpu_lib, dtype):
    splat = gpu_lib
    B, H, heads, page, d = 5000, 40, 16, 4, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn((B, h, 1, d), generator=g, device="cuda").to(dtype) for h in (H, heads, heads))
    kc, vc = (torch.zeros((B, heads, page, d), dtype=dtype, device="cuda") for _ in range(2))
    table = torch.randperm(B, generator=g, device="cuda").int()[:, None].contiguous()
    start = torch.arange(B, device="cuda", dtype=torch.int32) % page
    rot = splat.Rotary(page, 64)
    qr = splat.cache_append(kc, vc, table, start, k, v, rot=rot, Q=q)
    wq, wk = splat.rotary(rot, q, k, positions=start[:, None].contiguous())
    want = [torch.zeros_like(kc), torch.zeros_like(vc)]
    want[0][table[:, 0].long(), :, start.long()] = wk[:, :, 0]
    want[1][table[:, 0].long(), :, start.long()] = v[:, :, 0]
    torch.cuda.synchronize()
    assert torch.equal(qr, wq) and torch.equal(kc, want[0]) and torch.equal(vc, want[1])


def test_too_many_heads_are_refused(gpu_lib):
    splat = gpu_lib
    rot = splat.Rotary(8, 16)
    x = torch.zeros((1, 1, 1, 64), device="cuda", dtype=torch.bfloat16).expand(1, 2 ** 20 + 1, 1, 64)
    with pytest.raises(splat.SplatError, match="heads"):
        splat.rotary(rot, x)
    y = splat.rotary(rot, x[:, 1:])
    torch.cuda.synchronize()
    assert y.shape[1] == 2 ** 20 and (y == 0).all()
