"""A rotation built with one axis takes its positions as one with several does,
[axes, B, T], and as one without axes does."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("restart", [False, True])
def test_one_axis(gpu_lib, restart, dtype):
    splat, B, T = gpu_lib, 2, 9
    rot = splat.Rotary(500, 64, axes=(32,), restart=restart)
    x, k = (torch.randn((B, h, T, 64), device="cuda").to(dtype) for h in (3, 2))
    pos = torch.randint(0, 500, (B, T), dtype=torch.int32, device="cuda")
    want = splat.rotary(rot, x, positions=pos)
    assert torch.equal(splat.rotary(rot, x, positions=pos[None].contiguous()), want)
    assert torch.equal(splat.rotary(rot, x, positions=pos.new_tensor(range(T)).expand(1, B, T).contiguous()), splat.rotary(rot, x))
    import paper_2407_16847_amd.autograd as sag
    leaf = x.clone().requires_grad_()
    sag.rotary(rot, leaf, pos[None].contiguous()).backward(x)
    assert torch.equal(leaf.grad, splat.rotary(rot, x, positions=pos, inverse=True))
    caches = []
    for p in (pos, pos[None].contiguous()):
        kc, vc = (torch.zeros((4, 2, 16, 64), dtype=dtype, device="cuda") for _ in range(2))
        table = torch.tensor([[0, 2], [1, 3]], dtype=torch.int32, device="cuda")
        q = splat.cache_append(kc, vc, table, torch.tensor([0, 5], dtype=torch.int32, device="cuda"), k, k, rot=rot, Q=x, positions=p)
        caches.append((kc, vc, q))
    for a, b in zip(*caches):
        assert torch.equal(a, b)
    for bad in (pos.expand(2, B, T).contiguous(), pos[None, :1].contiguous(), pos[None, None].contiguous(), pos[0], pos[None].long()):
        with pytest.raises((ValueError, TypeError, splat.SplatError)):
            splat.rotary(rot, x, positions=bad)
    two = splat.Rotary(500, 64, axes=(16, 16))
    for bad in (None, pos, pos[None].contiguous()):
        with pytest.raises((ValueError, TypeError, splat.SplatError)):
            splat.rotary(two, x, positions=bad)
