"""A transformer's feed-forward block in 8 bits, from the library's operators: the residual's
addition with the norm, the first product, the (gated) activation function and the second
product, each reading the codes that the one before it wrote."""
from __future__ import annotations

from typing import Optional

import torch

from . import cham


class FeedForward:
    """y = act(n W_in^T) W_out^T, or (act(n G^T) * (n U^T)) W_out^T where W_in [2 H, K] holds G
    above U (gated), with n = rms_norm(x + residual) * norm_weight.

    The weights ([H or 2 H, K] and [K, H], any float type, on the device) are brought to the block
    format once; pow2 takes scales that are powers of two, which the matrix instructions apply
    themselves; exact forms the products as block_linear's exact does.  The weights are quantized on the
    current stream: a call on another one has to wait for it."""

    def __init__(self, w_in: torch.Tensor, w_out: torch.Tensor, norm_weight: Optional[torch.Tensor] = None,
                 eps: float = 1e-6, act: int = cham.ACT_GELU, gated: bool = False, pow2: bool = False,
                 exact: bool = False):
        K, H = w_out.shape
        if w_in.shape != (2 * H if gated else H, K):
            raise ValueError(f"w_in must be [{2 * H if gated else H}, {K}], got {tuple(w_in.shape)}")
        self.K, self.H, self.gated, self.act, self.eps, self.pow2 = K, H, gated, act, eps, pow2
        self.exact = exact
        self.norm_weight = norm_weight
        self.w_in = cham.block_quantize_weights(w_in, pow2=pow2)
        self.w_out = cham.block_quantize_weights(w_out, pow2=pow2)

    def __call__(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None,
                 residual_out: Optional[torch.Tensor] = None, stream=None):
        """(y, h): the block's output in x's type, and h = x + residual (None without one)."""
        q, h = cham.rms_norm_quantize(x, self.norm_weight, self.eps, residual=residual, residual_out=residual_out,
                                      pow2=self.pow2, stream=stream)
        t = cham.block_linear(q, self.w_in, dtype=x.dtype, stream=stream, exact=self.exact)
        q = cham.gated_quantize(t[:, :self.H], t[:, self.H:] if self.gated else None, self.act, pow2=self.pow2,
                                stream=stream)
        return cham.block_linear(q, self.w_out, dtype=x.dtype, stream=stream, exact=self.exact), h
