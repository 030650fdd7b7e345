"""The training calls as differentiable functions.

    from paper_2407_16847_amd import autograd as sag
    Q, K = sag.rotary(rot, Q), sag.rotary(rot, K)
    O = sag.sparse_mhsa(acsr, Q, K, V, scale)      # acsr built with grad=True
    O.backward(dO)

The gradients are the library's backward calls and can be taken once (not
differentiated again); forward-mode tangents are refused. To capture a training
step into a graph, capture sparse_mhsa_fwd_lse, sparse_mhsa_bwd and rotary
themselves: they allocate nothing when given their outputs. A backward pass of
these functions refuses to be captured: torch would run the leaves' accumulation
on the stream of any eager graph of the same leaves that still lives, outside
the capture.
"""
from __future__ import annotations

from typing import Optional

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import Acsr, Rotary
from . import rotary as _rotary
from . import sparse_mhsa_bwd, sparse_mhsa_fwd, sparse_mhsa_fwd_lse

__all__ = ["sparse_mhsa", "rotary"]


def _not_captured() -> None:
    if torch.cuda.is_available() and torch.cuda.is_current_stream_capturing():
        raise RuntimeError("the backward pass of autograd functions is not captured into a graph; "
                           "capture sparse_mhsa_bwd and rotary(inverse=True) instead")


def _gradient(x: torch.Tensor) -> torch.Tensor:
    """x as the calls take it: contiguous and at 16 bytes, which a gradient behind a
    concatenation need not be."""
    x = x.contiguous()
    return x if x.data_ptr() % 16 == 0 else x.clone()


class _SparseMHSA(torch.autograd.Function):
    @staticmethod
    def forward(ctx, acsr, Q, K, V, scale):
        O, lse = sparse_mhsa_fwd_lse(acsr, Q, K, V, scale)
        ctx.save_for_backward(Q, K, V, O, lse)
        ctx.acsr, ctx.scale = acsr, scale
        return O

    @staticmethod
    @once_differentiable
    def backward(ctx, dO):
        _not_captured()
        Q, K, V, O, lse = ctx.saved_tensors
        dQ, dK, dV = sparse_mhsa_bwd(ctx.acsr, Q, K, V, O, lse, _gradient(dO), ctx.scale)
        return None, dQ, dK, dV, None


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, rot, X, positions):
        ctx.rot = rot
        ctx.save_for_backward(positions)
        return _rotary(rot, X, positions=positions)

    @staticmethod
    @once_differentiable
    def backward(ctx, dY):
        _not_captured()
        positions, = ctx.saved_tensors
        return None, _rotary(ctx.rot, _gradient(dY), positions=positions, inverse=True), None


def sparse_mhsa(acsr: Acsr, Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                scale: float, training: bool = False) -> torch.Tensor:
    """O = softmax_nz(scale * M (x) Q K^T) V with gradients for Q, K and V.  Without
    any to take this is sparse_mhsa_fwd, whose O in bf16 differs by roundings from
    that of the training forward; training=True takes the training forward there too.
    Set it where a pass is run without gradients first and again with them, as some
    activation checkpointing does: the layers behind then see the same O both times."""
    if any(forward_ad.unpack_dual(x).tangent is not None for x in (Q, K, V)):
        raise NotImplementedError("sparse_mhsa has no forward-mode derivative")
    if not (torch.is_grad_enabled() and (Q.requires_grad or K.requires_grad or V.requires_grad)):
        if training:
            return sparse_mhsa_fwd_lse(acsr, Q, K, V, scale)[0]
        return sparse_mhsa_fwd(acsr, Q, K, V, scale)
    if not acsr._info["grad"]:
        raise ValueError("gradients need a handle built with grad=True")
    return _SparseMHSA.apply(acsr, Q, K, V, float(scale))


def rotary(rot: Rotary, X: torch.Tensor, positions: Optional[torch.Tensor] = None) -> torch.Tensor:
    """X [B, H, T, d] rotated to its tokens' positions, with its gradient."""
    return _Rotary.apply(rot, X, positions)
