"""The differentiable functions around their calls: what they refuse and which of
the calls they make.  CPU only, the calls themselves replaced."""
import pytest
import torch
from torch.autograd import forward_ad

from paper_2407_16847_amd import autograd as sag


class Handle:
    _info = {"grad": 1}


@pytest.fixture
def calls(monkeypatch):
    """The calls made, by name."""
    made = []

    def fwd(a, Q, K, V, s):
        made.append("fwd")
        return Q.detach() * 1

    def fwd_lse(a, Q, K, V, s):
        made.append("fwd_lse")
        return Q.detach() * 1, Q.detach().sum(-1)

    def bwd(a, Q, K, V, O, lse, dO, s):
        made.append("bwd")
        return dO * 1, dO * 2, dO * 3

    def rotary(rot, X, positions=None, inverse=False):
        made.append("rotary")
        return X.detach() * 1

    for name, f in (("sparse_mhsa_fwd", fwd), ("sparse_mhsa_fwd_lse", fwd_lse), ("sparse_mhsa_bwd", bwd),
                    ("_rotary", rotary)):
        monkeypatch.setattr(sag, name, f)
    return made


def three(**kw):
    return [torch.randn(1, 2, 4, 64, **kw) for _ in range(3)]


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("grad", [False, True])
def test_tangents_are_refused(calls, which, grad):
    """A dual tensor does not come back without its tangent."""
    x = three()
    with forward_ad.dual_level():
        dual = list(x)
        dual[which] = forward_ad.make_dual(x[which], torch.ones_like(x[which]))
        if grad:
            dual[which - 1].requires_grad_()
        with pytest.raises(NotImplementedError):
            sag.sparse_mhsa(Handle, *dual, 1.0)
        with torch.no_grad(), pytest.raises(NotImplementedError):
            sag.sparse_mhsa(Handle, *dual, 1.0)
        with pytest.raises(NotImplementedError):
            sag.rotary(None, dual[which])
        sag.sparse_mhsa(Handle, *x, 1.0)       # without a tangent as ever
    assert "fwd" in calls or grad


def test_functional_tangents_are_refused(calls):
    q, k, v = three()
    with pytest.raises((NotImplementedError, RuntimeError)):
        torch.func.jvp(lambda t: sag.sparse_mhsa(Handle, t, k, v, 1.0), (q,), (q,))
    assert calls == []


def test_training_forward_without_gradients(calls):
    """training=True takes one forward in both modes."""
    x = three()
    sag.sparse_mhsa(Handle, *x, 1.0)
    sag.sparse_mhsa(Handle, *x, 1.0, training=True)
    leaf = three(requires_grad=True)
    with torch.no_grad():
        sag.sparse_mhsa(Handle, *leaf, 1.0, training=True)
    sag.sparse_mhsa(Handle, *leaf, 1.0, training=True)
    sag.sparse_mhsa(Handle, *leaf, 1.0)
    assert calls == ["fwd", "fwd_lse", "fwd_lse", "fwd_lse", "fwd_lse"]


def test_gradients_off_their_alignment(calls, monkeypatch):
    """A gradient arrives as its graph leaves it: contiguous but not at 16 bytes
    behind a concatenation, without strides behind a sum."""
    seen = []
    for name in ("sparse_mhsa_bwd", "_rotary"):
        f = getattr(sag, name)

        def check(*args, f=f, **kw):
            x = args[1] if kw.get("inverse") else args[6] if len(args) > 6 else None
            if x is not None:
                seen.append(x.clone())
                assert x.is_contiguous() and x.data_ptr() % 16 == 0
            return f(*args, **kw)

        monkeypatch.setattr(sag, name, check)
    for dtype in (torch.float32, torch.bfloat16):
        for call in (lambda q, k, v: sag.sparse_mhsa(Handle, q, k, v, 1.0), lambda q, k, v: sag.rotary(None, q)):
            x = three(requires_grad=True, dtype=dtype)
            one = torch.zeros(1, dtype=dtype, requires_grad=True)
            want = torch.randn(513, dtype=dtype)
            torch.cat((one, call(*x).flatten())).backward(want)
            assert torch.equal(seen.pop().flatten(), want[1:])
            call(*x).sum().backward()
            assert (seen.pop() == 1).all()
            call(*x).transpose(1, 2).backward(want[1:].view(1, 4, 2, 64))
            assert torch.equal(seen.pop(), want[1:].view(1, 4, 2, 64).transpose(1, 2))
    assert not seen
