"""The norms around a block and their gradients in 64 bits, each with a bound on the error of a computation in 32 bits.

The bounds add up, to first order, what every rounding can contribute: u = 2^-24 for an operation, (length of the longest chain
of additions) u relative to the sum of absolute values for a sum, and half a step of the output's type for its last rounding.
The longest chain of a sum over a row: at most max(64, h / 64) terms in a lane, 32 in the trees over a workgroup.  Sums over
tokens are bounded by a chain of all of them.
"""
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def chain(h):
    return (max(64, h / 64) + 32) * U


def rounded(value, error, dtype):
    """The bound after the rounding to `dtype` (and below the smallest normal number)."""
    return error + HALF[dtype] * (value.abs() + error) + 2e-38


def mean(v):
    return v.mean(1, keepdim=True)


def f64(t):
    return None if t is None else t.detach().double()


def gate_rows(gate, N):
    """The gate's row of every token, in 64 bits (1 without a gate)."""
    return 1.0 if gate is None else f64(gate).repeat_interleave(N // gate.shape[0], 0)


def vector(t, like, absent):
    return torch.full_like(like[0], absent) if t is None else f64(t)


def forward(x, y=None, gate=None, w=None, b=None, w_post=None, b_post=None, scale=1.0, eps=1e-5, post=False, center=False):
    """{output: (value, bound on the error)} with r and H unrounded; the bounds of r and H include their rounding."""
    dtype, (N, h) = x.dtype, x.shape
    x = f64(x)
    c = chain(h)
    m1, rho1 = torch.zeros_like(x[:, :1]), torch.ones_like(x[:, :1])
    E_m1, E_rho1 = m1.clone(), m1.clone()
    r, E_r = x, torch.zeros_like(x)
    if y is not None:
        u, E_u = f64(y), torch.zeros_like(x)
        if post:
            v, wp, bp = u, vector(w_post, x, 1.0), vector(b_post, x, 0.0)
            if center:
                m1 = mean(v)
                E_m1 = c * mean(v.abs()) + U * m1.abs()
            rho1 = 1 / (mean((v - m1) ** 2) + eps).sqrt()
            # relative: the sum of squares (each with three roundings), and the error of the mean in it
            E_rho1 = c + 6 * U + mean((v - m1).abs()) * E_m1 * rho1 ** 2 + E_m1 ** 2 * rho1 ** 2
            vh = (v - m1) * rho1
            E_vh = rho1 * (E_m1 + U * (v - m1).abs()) + vh.abs() * (E_rho1 + U)
            u = vh * wp + bp
            E_u = wp.abs() * E_vh + 3 * U * ((vh * wp).abs() + bp.abs())
        f = scale * gate_rows(gate, N)
        f = f if isinstance(f, torch.Tensor) else torch.full_like(x[:1, :1], f)
        r = x + f * u
        E_r = f.abs() * E_u + 4 * U * (x.abs() + (f * u).abs())
    m2, E_m2 = torch.zeros_like(x[:, :1]), torch.zeros_like(x[:, :1])
    if center:
        m2 = mean(r)
        E_m2 = c * mean(r.abs()) + mean(E_r) + U * m2.abs()
    rho2 = 1 / (mean((r - m2) ** 2) + eps).sqrt()
    E_v = E_r + E_m2 + U * (r - m2).abs()
    E_rho2 = c + 6 * U + mean((r - m2).abs() * E_v) * rho2 ** 2 + mean(E_v ** 2) * rho2 ** 2
    rh = (r - m2) * rho2
    wv, bv = vector(w, x, 1.0), vector(b, x, 0.0)
    H = rh * wv + bv
    E_H = wv.abs() * (rho2 * E_v + rh.abs() * (E_rho2 + U)) + 3 * U * ((rh * wv).abs() + bv.abs())
    stats = torch.cat([m1, rho1, m2, rho2], 1).t()
    E_stats = torch.cat([E_m1, rho1 * E_rho1, E_m2, rho2 * E_rho2], 1).t() + 2e-38
    return {"r": (r, rounded(r, E_r, dtype)), "H": (H, rounded(H, E_H, dtype)), "stats": (stats, E_stats)}


def backward(dH, r, y, stats, dr=None, gate=None, w=None, w_post=None, b_post=None, scale=1.0, post=False, center=False,
             grad_dtype=torch.float32):
    """{gradient: (value, bound)}; gradients of activations are rounded to grad_dtype."""
    N, h = r.shape
    c, t = chain(h), (N + 16) * U
    dH, r, dr = f64(dH), f64(r), torch.zeros_like(r, dtype=torch.float64) if dr is None else f64(dr)
    m1, rho1, m2, rho2 = f64(stats).reshape(4, N, 1)
    a, rh = dH * vector(w, r, 1.0), (r - m2) * rho2
    ma = mean(a) if center else torch.zeros_like(m1)
    mar = mean(a * rh)
    dx = dr + rho2 * (a - ma - rh * mar)
    E = rho2 * (c * mean(a.abs()) * bool(center) + rh.abs() * (c + 6 * U) * mean((a * rh).abs())
                + 6 * U * (a.abs() + ma.abs() + (rh * mar).abs())) + 2 * U * (dr.abs() + dx.abs())
    out = {"dx": (dx, rounded(dx, E, grad_dtype)),
           "dw": ((dH * rh).sum(0), (t + 4 * U) * (dH * rh).abs().sum(0)), "db": (dH.sum(0), t * dH.abs().sum(0))}
    if y is None:
        return out
    yh = (f64(y) - m1) * rho1
    f = scale * gate_rows(gate, N)
    d = f * dx
    E_d = (abs(f) if not isinstance(f, torch.Tensor) else f.abs()) * E + 3 * U * d.abs()
    wp, bp = vector(w_post, r, 1.0), vector(b_post, r, 0.0)
    if gate is not None:
        u = yh * wp + bp if post else f64(y)
        E_u = 4 * U * ((yh * wp).abs() + bp.abs()) if post else 0.0
        part, E_part = scale * u * dx, abs(scale) * (u.abs() * E + E_u * dx.abs())

        def rows(v):
            return v.reshape(gate.shape[0], -1, h).sum(1)
        out["dgate"] = (rows(part), rows(E_part) + (t + 4 * U) * rows(part.abs()))
    if not post:
        out["dy"] = (d, rounded(d, E_d, grad_dtype))
        return out
    out["dw_post"] = ((d * yh).sum(0), (E_d * yh.abs()).sum(0) + (t + 4 * U) * (d * yh).abs().sum(0))
    out["db_post"] = (d.sum(0), E_d.sum(0) + t * d.abs().sum(0))
    k, E_k = d * wp, wp.abs() * E_d + U * (d * wp).abs()
    mk = mean(k) if center else torch.zeros_like(m1)
    mky = mean(k * yh)
    dy = rho1 * (k - mk - yh * mky)
    E_y = rho1 * (E_k + bool(center) * (mean(E_k) + c * mean(k.abs()))
                  + yh.abs() * (mean(E_k * yh.abs()) + (c + 6 * U) * mean((k * yh).abs()))
                  + 6 * U * (k.abs() + mk.abs() + (yh * mky).abs()))
    out["dy"] = (dy, rounded(dy, E_y, grad_dtype))
    return out


def check(name, got, value, bound):
    assert got.shape == value.shape, (name, got.shape, value.shape)
    off = (got.double() - value).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        at = tuple(int(i) for i in torch.nonzero(bad)[0])
        raise AssertionError("%s: %d of %d outside the bound, first at %s: got %r, expected %r, bound %r" % (
            name, int(bad.sum()), bad.numel(), at, float(got[at]), float(value[at]), float(bound[at])))
