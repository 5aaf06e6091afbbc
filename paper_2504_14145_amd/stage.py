"""One layer block of a pipeline stage, run with the stage operators.

The block is what the cost tables count as a layer norm and two matrix products
(the MLP half of a transformer layer, DIP arXiv 2504.14145 Sec. 6.1):

    n = layer_norm(x);  u = act(n w1^T + b1);  y = x + D(u w2^T + b2)

(of a language model whose MLP is gated, the block is the plain product of the same
sizes: the gate is not among the operators)

A forward keeps its activations or, under a memory strategy that recomputes
(Sec. 5.3), only its input; the backward then runs the forward again and draws
the same dropout mask, which is a function of the layer, the sample's seed and
the row.  A piece of a sample (Sec. 4) passes the row it starts at, so pieces
draw what the whole sample would.  Weight gradients are summed in float32 over
the pieces and microbatches of an iteration.  Everything runs on torch's
current stream.
"""
from __future__ import annotations

import math

from . import ops


class Block:
    """Weights [ffn, hidden] and [hidden, ffn] of float16 or bfloat16 and their
    float32 gradients; ``tp`` divides ffn among tensor-parallel ranks.  ``rank``'s
    share is held here, and the sums over ranks of y, dx and the gradients of gamma
    and beta are the caller's: rank 0's y has the residual and b2, its dx what came
    along the residual, and only it has a gradient of b2.  Weights are drawn from
    ``seed``: ranks give seeds of their own."""

    def __init__(self, hidden: int, ffn: int, act: str = "gelu", p: float = 0.0, layer: int = 0,
                 tp: int = 1, dtype=None, device="cuda", seed: int = 0, rank: int = 0):
        import torch
        if ffn % tp:
            raise ValueError(f"ffn {ffn} is not divisible by tp {tp}")
        if not 0 <= rank < tp:
            raise ValueError(f"rank {rank} is not one of {tp}")
        self.first = rank == 0
        self.hidden, self.ffn, self.act, self.p, self.layer = hidden, ffn // tp, act, p, layer
        dtype = torch.bfloat16 if dtype is None else dtype
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(shape, generator=g, device=device) * scale).to(dtype)

        self.w1 = normal(self.ffn, hidden, scale=1 / math.sqrt(hidden))
        self.w2 = normal(hidden, self.ffn, scale=1 / math.sqrt(self.ffn))
        self.b1 = torch.zeros(self.ffn, dtype=dtype, device=device)
        self.b2 = torch.zeros(hidden, dtype=dtype, device=device)
        self.gamma = torch.ones(hidden, dtype=dtype, device=device)
        self.beta = torch.zeros(hidden, dtype=dtype, device=device)
        self.grads = {n: torch.zeros(getattr(self, n).shape, device=device)
                      for n in ("w1", "b1", "w2", "b2", "gamma", "beta")}

    def _dropout(self, seed, row0):
        return ops.Dropout(self.p, seed, offset=self.layer, row0=row0) if self.p else None

    def forward(self, x, seed: int = 0, row0: int = 0, keep: bool = True):
        """(y, saved) for x [tokens, hidden]: rows row0 .. of the sample ``seed``."""
        import torch
        t = x.shape[0]
        n, mean, rstd = ops.group_norm(x.unsqueeze(1), 1, self.gamma, self.beta)
        n = n.squeeze(1)
        pre = torch.empty((t, self.ffn), dtype=x.dtype, device=x.device) \
            if keep and self.act != "none" else None
        u = ops.linear(n, self.w1, self.b1, act=self.act, pre=pre)
        y = ops.linear(u, self.w2, self.b2 if self.first else None, dropout=self._dropout(seed, row0),
                       residual=x if self.first else None)
        return y, (x, seed, row0, (n, mean, rstd, pre, u) if keep else None)

    def backward(self, dy, saved):
        """The gradient of x; those of the parameters are added to ``grads``."""
        x, seed, row0, kept = saved
        if kept is None:
            kept = self.forward(x, seed, row0)[1][3]
        n, mean, rstd, pre, u = kept
        g = self.grads
        du, _, _ = ops.linear_backward(dy, u, self.w2, dropout=self._dropout(seed, row0),
                                       dw=g["w2"], db=g["b2"] if self.first else None, bias=self.first,
                                       accumulate=True)
        dn, _, _ = ops.linear_backward(du, n, self.w1, act=self.act, pre=pre, dw=g["w1"],
                                       db=g["b1"], accumulate=True)
        dx, _, _ = ops.group_norm_backward(dn.unsqueeze(1), x.unsqueeze(1), mean, rstd, 1, self.gamma, self.beta,
                                           dgamma=g["gamma"], dbeta=g["beta"], accumulate=True)
        dx = dx.squeeze(1)
        return ops.dropout_add(dx, ops.Dropout(0.0, 0), residual=dy) if self.first else dx
