"""Plain 64-bit forms of the stage operators (TEST INFRASTRUCTURE ONLY), on the
CPU, and the error bounds that their float32 kernels have to keep.

Bounds: an output is rounded once, u |value| with the type's unit roundoff u
(and half its smallest subnormal); a float32 sum of n products in any order is
within (n + 8) 2^-24 sum |a b| of the sum, factor 2 for the products' and the
order's higher terms; an activation or its slope adds 2e-6 of its argument's
scale, and passes an error on by at most 1.2 times.
"""
import math

import torch

EPS32 = 2.0 ** -24
U = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126}
MASK32 = 0xFFFFFFFF


def philox(counter, key):
    """Philox4x32-10 of one counter, in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & MASK32, (p0 >> 32) ^ c[3] ^ k[1], p0 & MASK32]
        k = [(k[0] + 0x9E3779B9) & MASK32, (k[1] + 0xBB67AE85) & MASK32]
    return c


def mask(drop, m, n):
    """The kept elements of an m x n array (bool), counter by counter."""
    keep = torch.ones((m, n), dtype=torch.bool)
    if not drop.drop_of:
        return keep
    key = (drop.seed & MASK32, drop.seed >> 32)
    for i in range(m):
        for b in range((n + 7) // 8):
            w = philox((b, drop.row0 + i, drop.offset & MASK32, drop.offset >> 32), key)
            for j in range(min(8, n - 8 * b)):
                u = (w[j // 2] >> (16 * (j % 2))) & 0xFFFF
                keep[i, 8 * b + j] = u >= drop.drop_of
    return keep


def logistic(z):
    e = torch.exp(-z.abs())
    return torch.where(z >= 0, 1 / (1 + e), e / (1 + e))


def act(z, name):
    if name == "none":
        return z.clone()
    if name == "relu":
        return torch.clamp_min(z, 0)
    if name == "silu":
        return z * logistic(z)
    return z * logistic(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))


def slope(z, name):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).double()
    if name == "silu":
        e = logistic(z)
        return e * (1 + z * (1 - e))
    a = math.sqrt(2 / math.pi)
    e = logistic(2 * a * (z + 0.044715 * z ** 3))
    return e * (1 + z * (1 - e) * 2 * a * (1 + 3 * 0.044715 * z ** 2))


def dot_bound(n, magnitude):
    return 2 * (n + 8) * EPS32 * magnitude


def assert_close(got, want, bound, dtype, what):
    """|got - want| <= bound + the rounding to dtype, element by element."""
    got, want = got.detach().cpu().double(), want.cpu()
    limit = bound + U[dtype] * (want.abs() + bound) + TINY[dtype]
    off = (got - want).abs()
    assert got.shape == want.shape, what
    assert not torch.isnan(got).any(), f"{what}: NaN"
    bad = off > limit
    if bad.any():
        i = int(torch.argmax((off - limit).flatten()))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound; worst at {i}: "
                             f"{got.flatten()[i]} for {want.flatten()[i]}, bound {limit.flatten()[i]}")


class Linear:
    """Forward and gradients with their bounds, from CPU tensors of any type."""

    def __init__(self, x, w, bias, residual, act_name, drop, keep=None):
        self.x, self.w = x.cpu().double(), w.cpu().double()
        m, n, k = x.shape[0], w.shape[0], x.shape[1]
        self.name, self.scale = act_name, drop.scale if drop is not None and drop.drop_of else 1.0
        self.keep = keep if keep is not None else (
            mask(drop, m, n) if drop is not None else torch.ones((m, n), dtype=torch.bool))
        self.z = self.x @ self.w.T
        mag = self.x.abs() @ self.w.abs().T
        if bias is not None:
            self.z = self.z + bias.cpu().double()
            mag = mag + bias.cpu().double().abs()
        self.z_bound = dot_bound(k, mag)
        self.y = torch.where(self.keep, act(self.z, act_name) * self.scale, 0.0)
        self.y_bound = torch.where(self.keep, self.scale * (1.2 * self.z_bound + 2e-6 * self.z.abs()), 0.0)
        if residual is not None:
            r = residual.cpu().double()
            self.y = self.y + r
            self.y_bound = self.y_bound + 2 * EPS32 * (self.y.abs() + r.abs())

    def grads(self, dy, pre, dtype):
        """{name: (value, bound)} of dx, dw, db for the stored pre (None: no activation)."""
        m, n, k = self.x.shape[0], self.w.shape[0], self.x.shape[1]
        s = slope(pre.cpu().double(), self.name) if self.name != "none" else torch.ones((m, n), dtype=torch.double)
        d = torch.where(self.keep, dy.cpu().double() * self.scale, 0.0)
        g = d * s
        g32 = d.abs() * 4e-6 * (1 + (pre.cpu().double().abs() if self.name != "none" else 0)) \
            if self.name != "none" else 2 * EPS32 * d.abs()
        rounded = self.name != "none" or self.scale != 1.0
        g16 = g32 + (U[dtype] * (g.abs() + g32) + TINY[dtype] if rounded else 0)
        return {"dx": (g @ self.w, g16 @ self.w.abs() + dot_bound(n, (g.abs() + g16) @ self.w.abs())),
                "dw": (g.T @ self.x, g16.T @ self.x.abs() + dot_bound(m, (g.abs() + g16).T @ self.x.abs())),
                "db": (g.sum(0), g32.sum(0) + dot_bound(m, g.abs().sum(0)))}


class GroupNorm:
    """x [b, s, c] on the CPU, any type."""

    def __init__(self, x, groups, gamma, beta, eps, act_name):
        b, s, c = x.shape
        self.shape, self.groups, self.name = (b, s, c), groups, act_name
        self.per = c // groups
        v = self.split(x.cpu().double())
        n = s * self.per
        self.n = n
        self.mean = v.mean(2, keepdim=True)
        d = v - self.mean
        self.var = (d * d).mean(2, keepdim=True)
        self.rstd = 1 / torch.sqrt(self.var + eps)
        self.xh = d * self.rstd
        self.gamma = self.spread(gamma.cpu().double()) if gamma is not None else torch.ones_like(v)
        self.beta = self.spread(beta.cpu().double()) if beta is not None else torch.zeros_like(v)
        self.z = self.xh * self.gamma + self.beta
        # statistics: sums of n terms (of values shifted by one of them or by the
        # mean) relative to the spread of the values, seen through rstd; the values
        # themselves bring eps32 |x| rstd
        spread = torch.sqrt((d * d).mean(2, keepdim=True)) * self.rstd
        big = d.abs().amax(2, keepdim=True) * self.rstd
        chain = 2 * (min(n, 4096) + 8) * EPS32
        self.xh_bound = chain * (spread + 2 * big * big.clamp(max=4) / 4 + self.xh.abs()) + \
            4 * EPS32 * (v.abs() + self.mean.abs()) * self.rstd
        self.y = self.join(act(self.z, act_name))
        self.y_bound = self.join(1.2 * (self.xh_bound * self.gamma.abs() + 4 * EPS32 * (self.z.abs() + self.beta.abs()))
                                 + 2e-6 * self.z.abs())

    def split(self, v):
        b, s, c = self.shape
        return v.reshape(b, s, self.groups, self.per).permute(0, 2, 1, 3).reshape(b, self.groups, -1)

    def join(self, v):
        b, s, c = self.shape
        return v.reshape(b, self.groups, s, self.per).permute(0, 2, 1, 3).reshape(b, s, c)

    def spread(self, p):
        b, s, c = self.shape
        return self.split(p.reshape(1, 1, c).expand(b, s, c))

    def grads(self, dy):
        """{name: (value, bound)}; the bound takes mean and rstd as float32 statistics."""
        b, s, c = self.shape
        dv = self.split(dy.cpu().double())
        sl = slope(self.z, self.name)
        g = dv * sl
        zb = self.xh_bound * self.gamma.abs() + 4 * EPS32 * (self.z.abs() + self.beta.abs())
        gb = dv.abs() * (1.2 * zb + 4e-6 * (1 + self.z.abs())) if self.name != "none" else 2 * EPS32 * dv.abs()
        h, hb = g * self.gamma, gb * self.gamma.abs() + 2 * EPS32 * (g * self.gamma).abs()
        mean = lambda v: v.mean(2, keepdim=True)  # noqa: E731
        m1, m2 = mean(h), mean(h * self.xh)
        chain = 2 * (min(self.n, 4096) + 8) * EPS32
        m1b = mean(hb) + chain * mean(h.abs())
        hxb = hb * self.xh.abs() + h.abs() * self.xh_bound
        m2b = mean(hxb) + chain * mean((h * self.xh).abs())
        dx = self.rstd * (h - m1 - self.xh * m2)
        parts = h.abs() + m1.abs() + (self.xh * m2).abs()
        rel = self.xh_bound.amax(2, keepdim=True).clamp(max=1e-2)
        dxb = self.rstd * (hb + m1b + self.xh.abs() * m2b + self.xh_bound * m2.abs() + (8 * EPS32 + rel) * parts)
        many = 2 * (min(b * s, 4096) + 8) * EPS32
        gx = g * self.xh
        gxb = gb * self.xh.abs() + g.abs() * self.xh_bound
        total = lambda v: self.join(v).sum((0, 1))  # noqa: E731
        return {"dx": (self.join(dx), self.join(dxb)),
                "dgamma": (total(gx), total(gxb) + many * total(gx.abs())),
                "dbeta": (total(g), total(gb) + many * total(g.abs()))}
