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
