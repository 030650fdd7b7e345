"""The differentiable functions in use: activation checkpointing."""
import pytest
import torch
from torch.utils.checkpoint import checkpoint

from test_gpu_grad import TYPES, inputs, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("reentrant", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_a_checkpointed_layer(gpu_lib, d, dtype, reentrant):
    """The recomputed O is the first one bit for bit, and so are the gradients of a
    layer that is checkpointed and of one that is not."""
    from paper_2407_16847_amd import autograd as sag
    splat = gpu_lib
    a, _ = make(splat, "window_global", {"w": 40, "n_global": 5}, 450)
    x = [t.cuda() for t in inputs(450, d, 3, dtype, 3)]
    dO, x = x[3], x[:3]
    seen = []

    def layer(q, k, v):
        O = sag.sparse_mhsa(a, q, k, v, 0.125, training=True)
        seen.append(O.detach().clone())
        return O * O

    grads = []
    for wrap in (False, True):
        leaf = [t.clone().requires_grad_() for t in x]
        out = checkpoint(layer, *leaf, use_reentrant=reentrant) if wrap else layer(*leaf)
        out.backward(dO)
        grads.append([t.grad for t in leaf])
    torch.cuda.synchronize()
    assert len(seen) == 3 and all(torch.equal(seen[0], o) for o in seen)
    assert all(torch.equal(u, v) for u, v in zip(*grads))


@pytest.mark.parametrize("which", ["rotary", "append", "decode", "fwd_lse", "bwd"])
def test_a_call_into_a_saved_tensor_is_noticed(gpu_lib, which):
    """A call that writes into a tensor which a backward pass still needs: that pass
    raises instead of taking what the call has left there."""
    from paper_2407_16847_amd import autograd as sag
    splat = gpu_lib
    L, page, d = 48, 16, 64
    a, _ = make(splat, "window", {"w": 9}, L)
    rot = splat.Rotary(L, 32)
    q, k, v, dO = (t.cuda() for t in inputs(L, d, 2, torch.float32, 3))
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    table = torch.zeros((1, 3), dtype=torch.int32, device="cuda")
    lse = torch.zeros((1, 2, L), device="cuda")
    x = torch.zeros((1, 2, page, d) if which == "append" else (1, 2, 1, d) if which == "decode" else q.shape,
                    device="cuda")
    cache = torch.zeros((1, 2, page, d), device="cuda")
    new = torch.zeros((1, 2, 4, d), device="cuda")
    calls = {"rotary": lambda: splat.rotary(rot, x, Y=x),
             "append": lambda: splat.cache_append(x, cache, table, at, new, new),
             "decode": lambda: splat.sparse_mhsa_decode(a, new[:, :, :1].contiguous(), cache, cache.clone(), table,
                                                        at, 1.0, O=x),
             "fwd_lse": lambda: splat.sparse_mhsa_fwd_lse(a, q, k, v, 0.1, O=x, lse=lse),
             "bwd": lambda: splat.sparse_mhsa_bwd(a, q, k, v, q, lse, dO, 0.1, dQ=x)}
    leaf = torch.ones_like(x, requires_grad=True)
    (leaf * x).sum().backward()
    y = (leaf * x).sum()
    calls[which]()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():          # tensors without a version
        x = x.clone()
        calls[which]()
    torch.cuda.synchronize()
    out = sag.sparse_mhsa(a, q.requires_grad_(), k, v, 0.1)
    out.backward(dO)                      # and new outputs of the calls are no such writes
    torch.cuda.synchronize()
    assert torch.isfinite(q.grad).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_off_their_alignment(gpu_lib, dtype):
    """The gradients behind a concatenation are those of the pass without it."""
    from paper_2407_16847_amd import autograd as sag
    splat = gpu_lib
    a, _ = make(splat, "window", {"w": 20}, 100)
    rot = splat.Rotary(100, 64)
    x = [t.cuda() for t in inputs(100, 64, 2, dtype, 3)]
    dO, x = x[3], x[:3]
    grads = []
    for cat in (False, True):
        leaf = [t.clone().requires_grad_() for t in x]
        for k, call in ((3, lambda: sag.sparse_mhsa(a, *leaf, 0.125)), (1, lambda: sag.rotary(rot, leaf[0]))):
            out = call().flatten()
            want = dO.flatten()
            if cat:
                one = torch.zeros(1, dtype=dtype, device="cuda", requires_grad=True)
                out, want = torch.cat((one, out)), torch.cat((one.detach(), want))
            grads.append(torch.autograd.grad(out, leaf[:k], want))
    torch.cuda.synchronize()
    for got, ref in zip(grads[2:], grads[:2]):
        assert all(torch.equal(u, v) for u, v in zip(got, ref))
