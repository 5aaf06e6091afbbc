"""Layer blocks of a pipeline stage, run with the stage operators.

Block is what the cost tables count as a norm and two matrix products (the MLP
half of a transformer layer, DIP arXiv 2504.14145 Sec. 6.1):

    n = norm(x);  u = act(n w1^T + b1);  y = x + D(u w2^T + b2)

(of a language model whose MLP is gated, the block is the plain product of the same
sizes: the gate is not among the operators)

Projection is the start of the attention half, up to its heads:

    t = x + residual;  n = rms_norm(t);  q, k, v = n w^T + b;  q, k = rotary(q, k)

A forward keeps its activations, keeps them in 8 bits (33 / 64 of the memory of 16, and of
an MLP, whose pre then serves as u too, down to half of that; gradients of weights see
them rounded to four significant bits) or, under a
memory strategy that recomputes (Sec. 5.3), only its input; the backward then runs
the forward again and draws the same dropout mask, which is a function of the layer,
the sample's seed and the row.  A piece of a sample (Sec. 4) passes the row it starts at, so pieces
draw what the whole sample would.  Weight gradients are summed in float32 over
the pieces and microbatches of an iteration.  Everything runs on torch's
current stream.
"""
from __future__ import annotations

import math

from . import ops


KEEP = (True, 8, False)   # activations of the type, in 8 bits, none


def _known_keep(keep):
    if keep not in KEEP:
        raise ValueError(f"keep {keep!r} is not one of {KEEP}")


class Block:
    """Weights [ffn, hidden] and [hidden, ffn] of float16 or bfloat16 and their
    float32 gradients, behind a layer norm or, ``norm`` "rms", a root-mean-square norm
    (no beta); ``tp`` divides ffn among tensor-parallel ranks.  ``rank``'s
    share is held here, and the sums over ranks of y, dx and the gradients of gamma
    and beta are the caller's: rank 0's y has the residual and b2, its dx what came
    along the residual, and only it has a gradient of b2.  Weights are drawn from
    ``seed``: ranks give seeds of their own."""

    def __init__(self, hidden: int, ffn: int, act: str = "gelu", p: float = 0.0, layer: int = 0,
                 tp: int = 1, dtype=None, device="cuda", seed: int = 0, rank: int = 0,
                 norm: str = "layer"):
        import torch
        if norm not in ("layer", "rms"):
            raise ValueError(f"norm {norm!r} is neither layer nor rms")
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
        self.beta = torch.zeros(hidden, dtype=dtype, device=device) if norm == "layer" else None
        self.grads = {n: torch.zeros(getattr(self, n).shape, device=device)
                      for n in ("w1", "b1", "w2", "b2", "gamma") + (("beta",) if norm == "layer" else ())}

    def _dropout(self, seed, row0):
        return ops.Dropout(self.p, seed, offset=self.layer, row0=row0) if self.p else None

    def forward(self, x, seed: int = 0, row0: int = 0, keep=True):
        """(y, saved) for x [tokens, hidden]: rows row0 .. of the sample ``seed``.
        ``keep``: True, 8 (in 8 bits) or False (nothing but x)."""
        import torch
        _known_keep(keep)
        t = x.shape[0]
        mean = n8 = None
        if self.beta is None:
            n, _, rstd, n8 = ops.rms_norm(x, self.gamma, packed=keep == 8)
        else:
            n, mean, rstd = ops.group_norm(x.unsqueeze(1), 1, self.gamma, self.beta)
            n = n.squeeze(1)
            if keep == 8:
                n8 = ops.pack8(n)
        pre = None
        if keep and self.act != "none":
            pre = ops.Packed8.empty(t, self.ffn, x.device) if keep == 8 else \
                torch.empty((t, self.ffn), dtype=x.dtype, device=x.device)
        u = ops.linear(n, self.w1, self.b1, act=self.act, pre=pre)
        y = ops.linear(u, self.w2, self.b2 if self.first else None, dropout=self._dropout(seed, row0),
                       residual=x if self.first else None)
        if keep == 8:       # u again from pre, or itself
            n, u = n8, ops.pack8(u) if pre is None else None
        return y, (x, seed, row0, (n, mean, rstd, pre, u) if keep else None)

    def backward(self, dy, saved):
        """The gradient of x; those of the parameters are added to ``grads``."""
        x, seed, row0, kept = saved
        if kept is None:
            kept = self.forward(x, seed, row0)[1][3]
        n, mean, rstd, pre, u = kept
        g = self.grads
        du, _, _ = ops.linear_backward(dy, pre if u is None else u, self.w2, dropout=self._dropout(seed, row0),
                                       dw=g["w2"], db=g["b2"] if self.first else None, bias=self.first,
                                       accumulate=True, x_act=self.act if u is None else "none")
        dn, _, _ = ops.linear_backward(du, n, self.w1, act=self.act, pre=pre, dw=g["w1"],
                                       db=g["b1"], accumulate=True)
        if self.beta is None:
            return ops.rms_norm_backward(dn, x, rstd, self.gamma, dtotal=dy if self.first else None,
                                         dgamma=g["gamma"], accumulate=True)[0]
        dx, _, _ = ops.group_norm_backward(dn.unsqueeze(1), x.unsqueeze(1), mean, rstd, 1, self.gamma, self.beta,
                                           dgamma=g["gamma"], dbeta=g["beta"], accumulate=True)
        dx = dx.squeeze(1)
        return ops.dropout_add(dx, ops.Dropout(0.0, 0), residual=dy) if self.first else dx


class Projection:
    """A weight [(heads + 2 keys) dim, hidden] of float16 or bfloat16, its bias, the
    norm's gamma and their float32 gradients.  ``sections``: the pairs of a head that
    turn with each axis of the positions (ops.rotary_frequencies has ``base`` and
    ``shared``).  Of ``tp`` tensor-parallel ranks each has its share of the heads, from a
    ``seed`` of its own; the sums over ranks of dx and gamma's gradient are the caller's,
    and only rank 0's dx has what came along the stream of residuals."""

    def __init__(self, hidden: int, heads: int, keys: int, dim: int, sections, base: float = 10000.0,
                 shared: bool = False, interleaved: bool = False, tp: int = 1, dtype=None, device="cuda",
                 seed: int = 0, rank: int = 0):
        import torch
        if heads % tp or keys % tp:
            raise ValueError(f"{heads} heads and {keys} of keys are not divisible by tp {tp}")
        if not 0 <= rank < tp:
            raise ValueError(f"rank {rank} is not one of {tp}")
        if 2 * sum(sections) > dim:
            raise ValueError(f"{sum(sections)} pairs in a head of {dim} elements")
        self.first = rank == 0
        self.heads, self.keys, self.dim, self.interleaved = heads // tp, keys // tp, dim, interleaved
        dtype = torch.bfloat16 if dtype is None else dtype
        rows = (self.heads + 2 * self.keys) * dim
        g = torch.Generator(device=device).manual_seed(seed)
        self.w = (torch.randn((rows, hidden), generator=g, device=device) / math.sqrt(hidden)).to(dtype)
        self.b = torch.zeros(rows, dtype=dtype, device=device)
        self.gamma = torch.ones(hidden, dtype=dtype, device=device)
        self.frequencies, self.axis = ops.rotary_frequencies(sections, base, shared, device)
        self.grads = {n: torch.zeros(getattr(self, n).shape, device=device) for n in ("w", "b", "gamma")}

    def _parts(self, qkv):
        """The heads of q, k and v in a product's output."""
        v = qkv.view(qkv.shape[0], self.heads + 2 * self.keys, self.dim)
        return v[:, :self.heads], v[:, self.heads:self.heads + self.keys], v[:, self.heads + self.keys:]

    def forward(self, x, positions, residual=None, keep=True):
        """(q, k, v, total, saved) for x [tokens, hidden] and positions [tokens, axes];
        ``keep`` as Block's."""
        _known_keep(keep)
        n, total, rstd, n8 = ops.rms_norm(x, self.gamma, residual=residual, packed=keep == 8)
        q, k, v = self._parts(ops.linear(n, self.w, self.b))
        ops.rotary(q, positions, self.frequencies, self.axis, k=k, interleaved=self.interleaved, out=q, out_k=k)
        return q, k, v, total, (total, positions, ((n8 if keep == 8 else n), rstd) if keep else None)

    def backward(self, dq, dk, dv, saved, dtotal=None):
        """The gradient of x and of the residual, for those of q, k, v and ``dtotal``, of
        total; those of the parameters are added to ``grads``."""
        import torch
        total, positions, kept = saved
        if kept is None:
            n, _, rstd, _ = ops.rms_norm(total, self.gamma)
        else:
            n, rstd = kept
        g = self.grads
        d = torch.empty((total.shape[0], self.w.shape[0]), dtype=total.dtype, device=total.device)
        to_q, to_k, to_v = self._parts(d)
        ops.rotary_backward(dq, positions, self.frequencies, self.axis, dk=dk, interleaved=self.interleaved,
                            out=to_q, out_k=to_k)
        to_v.copy_(dv)
        dn, _, _ = ops.linear_backward(d, n, self.w, dw=g["w"], db=g["b"], accumulate=True)
        return ops.rms_norm_backward(dn, total, rstd, self.gamma, dtotal=dtotal if self.first else None,
                                     dgamma=g["gamma"], accumulate=True)[0]
