"""The operators around the attention core in a block of a network, on torch tensors: rotary positions on q and k, and the norms of
the residual stream with its gates and scales.  Each has its gradients as a method of its own, like ``CastlingAttn.backward``: results have no
autograd history, whether or not the inputs require gradients, and a training step chains the methods by hand.  All
arithmetic is in the CUDA library.  Objects hold sizes and constants only: one serves any number of streams and threads.

A block as a user writes it (``norm`` of the block before gave ``y``):

    qkv = project(y).view(B, N, 3, H, d)
    q, k, v = (qkv[:, :, i].permute(0, 2, 1, 3) for i in range(3))
    q, k = rope.forward(q, k, grid=(gridH, gridW), prefix_tokens=1)
    out = attn.forward(q, k, v, dw_weight, dw_bias, gridH, gridW)
    x, y = norm.forward(x, output(out), weight=w, bias=b, scale=layer_scale, gate=gate)
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from . import attn as _attn   # binds the torch-facing module to the library
from . import binding as _b

_call = _attn._torch_call
_NORMS = {None: _b.NORM_NONE, "layer": _b.NORM_LAYER, "rms": _b.NORM_RMS}


class GridRope:
    """Rotary positions over one to three axes (time, height, width).

    ``axis_dims``: dimensions of a head that turn with each axis, even, one axis after the other from the first dimension on; what
    is behind them is left as it is.  Pair i of an axis with n dimensions turns by ``position * base ** (-2 i / n)``.
    ``interleaved``: a pair is two neighbouring elements; otherwise elements i and i + n / 2 of its axis.
    """

    def __init__(self, axis_dims: Sequence[int], base: float = 10000.0, interleaved: bool = False):
        dims = tuple(int(n) for n in axis_dims)
        if not 1 <= len(dims) <= 3 or any(n <= 0 or n % 2 for n in dims):
            raise ValueError("axis_dims: one to three positive even numbers")
        if not 0.0 < float(base) < float("inf"):
            raise ValueError("base must be positive")
        self.axis_dims, self.base, self.interleaved = dims, float(base), bool(interleaved)

    def forward(self, q, k: Optional[torch.Tensor] = None, grid: Optional[Tuple[int, ...]] = None, prefix_tokens: int = 0,
                positions: Optional[torch.Tensor] = None, inplace: bool = False) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """q ``[B, H, N, d]`` and k (its number of heads may be another; or None), any strides but nought, 1 in the last dimension,
        float32 or bfloat16.  Either ``grid``, a size per axis, last axis fastest: the positions of the token grid behind
        ``prefix_tokens`` leading tokens, which are copied; or ``positions``, int32, int64 or float32, ``[B, N, axes]``, ``[1, N, axes]``
        or ``[N, axes]``, contiguous: a decoded token's, say.  Returns new (q, k), or with ``inplace`` the same ones, turned, which
        must not share elements (slices of one tensor are fine, also with heads of their own)."""
        return self._turn(False, q, k, grid, prefix_tokens, positions, inplace)

    def backward(self, grad_q, grad_k: Optional[torch.Tensor] = None, grid: Optional[Tuple[int, ...]] = None, prefix_tokens: int = 0,
                 positions: Optional[torch.Tensor] = None, inplace: bool = False) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """Gradients of forward's inputs from those of its outputs: the opposite rotation."""
        return self._turn(True, grad_q, grad_k, grid, prefix_tokens, positions, inplace)

    def _turn(self, inverse, q, k, grid, prefix_tokens, positions, inplace):
        r = _call.rotate(self.axis_dims, self.base, self.interleaved, inverse, q, k, None if grid is None else tuple(grid), prefix_tokens,
                         positions, inplace)
        if r.__class__ is int:
            raise _b.CastlingError(r, "castling_attn_rotate")
        return r


class BlockNormGrads(NamedTuple):
    """Gradients in the order of ``BlockNorm.forward``'s arguments; None for what the call did not have."""
    x: torch.Tensor
    branch: Optional[torch.Tensor]
    weight: Optional[torch.Tensor]
    bias: Optional[torch.Tensor]
    post_weight: Optional[torch.Tensor]
    post_bias: Optional[torch.Tensor]
    scale: Optional[torch.Tensor]
    gate: Optional[torch.Tensor]


class BlockNorm:
    """The residual stream between two blocks:

        u = branch                                            or, with ``post``, norm(branch) * post_weight + post_bias
        h = residual_scale * x + gate[b] * scale * u          (without a branch: residual_scale * x)
        y = norm(h) * weight + bias

    ``kind`` is the norm that makes y: ``"layer"``, ``"rms"``, or None (behind the last block: h alone).  Parameters left out are
    factors of one and summands of nought.
    """

    def __init__(self, kind: Optional[str] = "layer", post: Optional[str] = None, eps: float = 1e-6, residual_scale: float = 1.0):
        if kind not in _NORMS or post not in _NORMS:
            raise ValueError("kind and post: 'layer', 'rms' or None")
        if not float(eps) > 0.0:
            raise ValueError("eps must be positive")
        self.kind, self.post, self.eps, self.residual_scale = kind, post, float(eps), float(residual_scale)
        self._head = (_NORMS[kind], _NORMS[post], self.eps, self.residual_scale)

    def forward(self, x, branch: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                gate: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
        """x and branch ``[B, N, D]`` (or ``[N, D]``: one sequence), any strides but nought, 1 in the last dimension, float32 or bfloat16; parameters
        ``[D]``, the gate ``[B, D]``, contiguous, of the same dtype.  Returns new contiguous (h, y); y is None without ``kind``, and h is x itself
        where there is no branch and residual_scale is 1."""
        r = _call.norm_forward(*self._head, x, branch, weight, bias, post_weight, post_bias, scale, gate)
        if r.__class__ is int:
            raise _b.CastlingError(r, "castling_attn_norm_forward")
        return r

    def backward(self, grad_y: Optional[torch.Tensor], grad_h: Optional[torch.Tensor], x, branch: Optional[torch.Tensor] = None,
                 weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, post_weight: Optional[torch.Tensor] = None,
                 post_bias: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                 gate: Optional[torch.Tensor] = None) -> BlockNormGrads:
        """Gradients of everything that forward was given (the same arguments again: neither h nor statistics need be kept) from those
        of y and h; either may be None.  Parameters' gradients are summed in fp32 and rounded once to the tensors' dtype."""
        r = _call.norm_backward(*self._head, x, branch, weight, bias, post_weight, post_bias, scale, gate, grad_y, grad_h)
        if r.__class__ is int:
            raise _b.CastlingError(r, "castling_attn_norm_backward")
        return BlockNormGrads(*r)
