"""A transformer's attention block in 8 bits, from the library's operators: the residual's addition
with the norm, the product that makes queries, keys and values, the heads' norm and rotation,
attention over the prompt itself or over a paged cache, and the output product."""
from __future__ import annotations

from typing import Optional

import torch

from . import cham


class AttentionBlock:
    """y = attention(q, k, v) W_out^T with the heads of (q, k, v) = n W_qkv^T, n = rms_norm(x +
    residual) * norm_weight; q and k are normed (where q_weight and k_weight are given) and turned (freq).

    x is float16 or bfloat16.  W_qkv [(heads + 2 kv_heads) D, K] and W_out [K, heads D] are brought to the
    block format once, on the current stream: a call on another one has to wait for it.  pow2 and exact are
    FeedForward's."""

    def __init__(self, w_qkv: torch.Tensor, w_out: torch.Tensor, heads: int, kv_heads: Optional[int] = None,
                 norm_weight: Optional[torch.Tensor] = None, q_weight: Optional[torch.Tensor] = None,
                 k_weight: Optional[torch.Tensor] = None, eps: float = 1e-6, freq: Optional[torch.Tensor] = None,
                 layout: int = cham.ROT_HALF, pow2: bool = False, exact: bool = False):
        kv_heads = heads if kv_heads is None else kv_heads
        K, N = w_out.shape
        if N % heads or w_qkv.shape != ((heads + 2 * kv_heads) * (N // heads), K):
            raise ValueError(f"w_qkv {tuple(w_qkv.shape)} and w_out {tuple(w_out.shape)} do not fit {heads} and {kv_heads} heads")
        if (q_weight is None) != (k_weight is None):
            raise ValueError("queries and keys are both normed, or neither")
        self.heads, self.kv_heads, self.D, self.eps, self.pow2, self.exact = heads, kv_heads, N // heads, eps, pow2, exact
        self.norm_weight, self.freq = norm_weight, freq
        self.how = dict(q_weight=q_weight, k_weight=k_weight, eps=eps, norm=q_weight is not None, freq=freq, layout=layout)
        self.w_qkv = cham.block_quantize_weights(w_qkv, pow2=pow2)
        self.w_out = cham.block_quantize_weights(w_out, pow2=pow2)

    def _heads(self, x, residual, residual_out, stream):
        n, h = cham.rms_norm_quantize(x, self.norm_weight, self.eps, residual=residual, residual_out=residual_out,
                                      pow2=self.pow2, stream=stream)
        t = cham.block_linear(n, self.w_qkv, dtype=x.dtype, stream=stream, exact=self.exact)
        t = t.view(x.shape[0], self.heads + 2 * self.kv_heads, self.D)
        return t[:, :self.heads], t[:, self.heads:self.heads + self.kv_heads], t[:, self.heads + self.kv_heads:], h

    def _out(self, o, x, stream):
        o = cham.gated_quantize(o.view(x.shape[0], self.heads * self.D), None, cham.ACT_NONE, pow2=self.pow2, stream=stream)
        return cham.block_linear(o, self.w_out, dtype=x.dtype, stream=stream, exact=self.exact)

    def __call__(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None,
                 residual_out: Optional[torch.Tensor] = None, *, positions: Optional[torch.Tensor] = None,
                 batch: Optional[int] = None, cu: Optional[torch.Tensor] = None, causal: bool = False, stream=None):
        """(y, h) of whole sequences: `batch` of equal lengths, or packed rows cu[b] .. cu[b + 1].  h = x +
        residual (None without one); positions int32 [T] where there is a rotation."""
        q, k, v, h = self._heads(x, residual, residual_out, stream)
        if self.how["norm"] or self.freq is not None or positions is not None:  # in place: the product's output is this call's own
            cham.norm_rotate(q, k, q_out=q, k_out=k, positions=positions, stream=stream, **self.how)
        o = cham.attention(q, k, v, batch=batch, cu_q=cu, causal=causal, stream=stream)
        return self._out(o, x, stream), h

    def step(self, x: torch.Tensor, cache: cham.Cache, slots: torch.Tensor, table: torch.Tensor, lens: torch.Tensor,
             residual: Optional[torch.Tensor] = None, residual_out: Optional[torch.Tensor] = None, *,
             positions: Optional[torch.Tensor] = None, cu: Optional[torch.Tensor] = None, stream=None):
        """(y, h) of the sequences' next tokens, one of each or rows cu[b] .. cu[b + 1] (a chunk of a prompt):
        their keys and values go to the slots of the cache, and they see their sequence's lens[b] tokens
        there, causally (see cham.cache_write and cham.cache_attention)."""
        q, k, v, h = self._heads(x, residual, residual_out, stream)
        cham.cache_write(cache, slots, k, v, q, q_out=q, positions=positions, stream=stream, **self.how)
        o = cham.cache_attention(q, cache, table, lens, cu, stream=stream)
        return self._out(o, x, stream), h
