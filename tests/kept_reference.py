"""Plain forms of the norm, the rotary positions and the 8-bit values (TEST
INFRASTRUCTURE ONLY), on the CPU, with the error bounds of their float32 kernels.

Bounds follow ops_reference: u |value| for an output's one rounding; a float32 sum of n
terms in any order is within 2 (n + 8) 2^-24 of the sum of their magnitudes (n counted
up to 4096: beyond, the sums are trees of parts).  A value in 8 bits is off by at most
half a step, 2^-4 of it (four significant bits), and not below half of 2^-9 scales.
"""
import torch

from ops_reference import EPS32, TINY, U, act

F8 = torch.float8_e4m3fn


def scale_bytes(v):
    """The scale's byte of each 32 columns of a float64 matrix, from the definition."""
    m, n = v.shape
    pad = torch.zeros((m, -n % 32), dtype=v.dtype)
    a = torch.cat((v, pad), 1).reshape(m, -1, 32).abs()
    most = torch.where(torch.isfinite(a), a, 0.0).amax(2)
    out = torch.empty(most.shape, dtype=torch.uint8)
    for i, x in enumerate(most.flatten().tolist()):
        e = -126
        if x > 0:
            while x > 448 * 2.0 ** e:
                e += 1
        out.view(-1)[i] = e + 127
    return out


def pack(x):
    """(values, scales) of a matrix of any type whose values are exact."""
    v = x.cpu().double()
    s = scale_bytes(v)
    scale = torch.pow(2.0, s.double() - 127).repeat_interleave(32, 1)[:, :v.shape[1]]
    q = v / scale                              # exact: a power of two
    q = torch.where(torch.isfinite(q), q, float("nan"))
    return round_e4m3(q).float().to(F8), s


def round_e4m3(q):
    """To nearest even with four significant bits and steps of at least 2^-9."""
    mag = q.abs().clamp_min(2.0 ** -6)
    step = torch.pow(2.0, torch.floor(torch.log2(mag)) - 3)
    return torch.round(q / step) * step


def unpack(values, scales):
    """The float64 values of a matrix in 8 bits."""
    scale = torch.pow(2.0, scales.cpu().double() - 127).repeat_interleave(32, 1)[:, :values.shape[1]]
    return values.cpu().float().double() * scale


def assert_kept(values, scales, want, bound, what):
    """A packed matrix whose float32 values were within bound of want."""
    got = unpack(values, scales)
    high, low = scale_bytes(want.abs() + bound), scale_bytes((want.abs() - bound).clamp_min(0))
    s = scales.cpu()
    assert bool(((s >= low) & (s <= high)).all()), f"{what}: scales"
    most = torch.pow(2.0, high.double() - 127).repeat_interleave(32, 1)[:, :want.shape[1]]
    limit = bound + 2.0 ** -4 * (want.abs() + bound) + 2.0 ** -10 * most
    off = (got - want).abs()
    assert bool((off <= limit).all()), f"{what}: {float((off - limit).max())} beyond the bound"


class RmsNorm:
    def __init__(self, x, residual, gamma, eps):
        self.total = x.cpu() if residual is None else (x.cpu().float() + residual.cpu().float()).to(x.dtype)
        t = self.total.double()
        self.gamma = torch.ones(t.shape[1], dtype=torch.double) if gamma is None else gamma.cpu().double()
        c = t.shape[1]
        self.rstd = 1 / torch.sqrt((t * t).mean(1) + eps) if c else torch.full((t.shape[0],), eps ** -0.5, dtype=torch.double)
        self.chain = 2 * (min(c, 4096) + 8) * EPS32
        # half of the mean's relative error, root, quotient and the row's last products
        self.rel = self.chain / 2 + 8 * EPS32
        self.xh = t * self.rstd[:, None]
        self.y = self.xh * self.gamma
        self.y_bound = self.rel * self.y.abs()

    def grads(self, dy, dtotal):
        dy = dy.cpu().double()
        m = dy.shape[0]
        h = dy * self.gamma
        hx = h * self.xh
        dot = hx.mean(1, keepdim=True)
        dotb = (self.chain + 2 * self.rel) * hx.abs().mean(1, keepdim=True)
        r = self.rstd[:, None]
        dx = r * (h - self.xh * dot)
        dxb = r * (self.xh.abs() * dotb + (8 * EPS32 + 3 * self.rel) * (h.abs() + (self.xh * dot).abs()))
        if dtotal is not None:
            dx = dx + dtotal.cpu().double()
            dxb = dxb + 2 * EPS32 * (dx.abs() + dtotal.cpu().double().abs())
        each = (dy * self.xh).abs().sum(0)
        many = 2 * (min(m, 4096) + 8) * EPS32
        return {"dx": (dx, dxb), "dgamma": ((dy * self.xh).sum(0), (many + self.rel) * each)}


def rotary(x, pos, freq, axis, interleaved, inverse=False):
    """(value, bound) of x [t, heads, dim] on the CPU.  Sine and cosine are off by two
    roundings and by their argument's, 2^-24 of at most a half turn; the two products and
    their sum by three more: within 2^-20 of the pair's magnitudes."""
    v = x.cpu().double()
    pairs = freq.shape[0]
    j = torch.arange(pairs)
    first = 2 * j if interleaved else j
    second = first + (1 if interleaved else pairs)
    p = pos.cpu().double().reshape(x.shape[0], -1)
    axis = axis.cpu().long()
    on = (axis >= 0) & (axis < p.shape[1])
    angle = torch.zeros((x.shape[0], pairs), dtype=torch.double)
    angle[:, on] = p[:, axis[on]] * freq.cpu()[on]
    c, s = angle.cos()[:, None], angle.sin()[:, None] * (-1 if inverse else 1)
    a, b = v[..., first], v[..., second]
    out, bound = v.clone(), torch.zeros_like(v)
    out[..., first], out[..., second] = a * c - b * s, a * s + b * c
    bound[..., first] = bound[..., second] = 2.0 ** -20 * (a.abs() + b.abs())
    return out, bound


def kept_x(values, scales, x_act, dtype):
    """(value, bound) of the x that a gradient takes from 8 bits."""
    z = unpack(values, scales)
    x = act(z, x_act)
    bound = TINY[dtype] + (0 if x_act == "none" else U[dtype] * x.abs() + 2e-6 * z.abs())
    return x, torch.zeros_like(x) + bound
