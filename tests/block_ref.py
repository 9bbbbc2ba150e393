"""Products with weights and norms between blocks in 64 bits on the CPU, each with a bound on what rounding may do to a kernel that
follows the same formulas in 32 bits and rounds its results once.

Half a step of a type is UNIT relative, or TINY absolute below its normal range.  A sum of n terms in 32 bits is off by at most
n * 2^-24 of the sum of its terms' magnitudes, in whatever order.
"""
import math

import torch

from attention_ref import UNIT, check  # noqa: F401

E = 2.0 ** -24
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -25}


def act(z, kind):
    """(activation, derivative, second derivative's largest magnitude nearby)."""
    if kind == "relu":
        return z.clamp(min=0), (z > 0).double()
    if kind == "gelu":
        p = 0.5 * torch.erfc(-z / 2 ** 0.5)
        return z * p, p + z * torch.exp(-z * z / 2) / (2 * math.pi) ** 0.5
    if kind == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    return z, torch.ones_like(z)


def linear(x, w, bias, kind, residual, dtype):
    """(out, bound, z, bound) from float64 inputs.  An activation's slope is at most 1.13; the functions that it is made of are
    off by 8 half steps of fp32 at most, relative to z."""
    K = x.shape[1]
    z, mass = x @ w.T, x.abs() @ w.abs().T
    if bias is not None:
        z, mass = z + bias, mass + bias.abs()
    ez = (K + 4) * E * mass
    a, _ = act(z, kind)
    ea = 1.13 * ez + 8 * E * z.abs()
    out = a if residual is None else a + residual
    eo = ea + 2 * E * out.abs()
    u, t = UNIT[dtype], TINY[dtype]
    return out, u * (out.abs() + eo) + eo + t, z, u * (z.abs() + ez) + ez + t


def linear_back(dout, x, w, z, kind, dtype):
    """((dx, bound), (dw, bound), (dbias, bound)).  The slope is made of functions that are off by 8 half steps, times |z| + 1."""
    M, N = dout.shape
    u, t = UNIT[dtype], TINY[dtype]
    if kind is None:
        dz, ez, er = dout, torch.zeros_like(dout), torch.zeros_like(dout)
    else:
        _, s = act(z, kind)
        dz = dout * s
        ez = dout.abs() * 8 * E * (z.abs() + 1) + E * dz.abs()           # not rounded to the type
        er = ez + u * (dz.abs() + ez) + t                                # rounded
    dx, dw, db = dz @ w, dz.T @ x, dz.sum(0)
    bx = er @ w.abs() + (N + 2) * E * ((dz.abs() + er) @ w.abs())
    bw = er.T @ x.abs() + (M + 2) * E * ((dz.abs() + er).T @ x.abs())
    bb = ez.sum(0) + (M + 2) * E * (dz.abs() + ez).sum(0)
    return [(v, b + u * (v.abs() + b) + t) for v, b in ((dx, bx), (dw, bw), (db, bb))]


def _norm(a, ea, eps, centred):
    """(n(a), bound, factor r, its relative bound): `a` is off by ea already."""
    C = a.shape[1]
    m = a.mean(1, keepdim=True) if centred else torch.zeros(a.shape[0], 1).double()
    em = ((C + 2) * E * a.abs().mean(1, keepdim=True) + ea.mean(1, keepdim=True)) if centred else 0 * m
    d = a - m
    ed = ea + em + E * (d.abs() + em)
    v = (d * d).mean(1, keepdim=True)
    ev = (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + (C + 3) * E * (v + (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True))
    r = (v + eps) ** -0.5
    rr = 0.5 * ev / (v + eps - ev).clamp(min=1e-300) + 4 * E                       # (1 + q)^-1/2 - 1 is at most q / 2 / (1 - q)
    n = d * r
    return n, (ed * r + n.abs() * rr + ed * r * rr) + 2 * E * n.abs(), r, rr


def norm(x, y, gate, post, pre, scale, eps, centred, norm_post, norm_pre, dtype):
    """(h, bound, z, bound), None for what there is not."""
    u, t = UNIT[dtype], TINY[dtype]
    h, eh, z, bz = x, torch.zeros_like(x), None, None
    if y is not None:
        v, ev = y, torch.zeros_like(y)
        if norm_post:
            v, ev = _norm(y, ev, eps, centred)[:2]
        for by in (post, gate):
            if by is not None:
                v, ev = v * by, ev * by.abs() + E * (v * by).abs()
        v, ev = scale * v, abs(scale) * ev + 2 * E * (scale * v).abs()
        h = x + v
        eh = ev + E * (h.abs() + ev)
    if norm_pre:
        n, en = _norm(h, eh, eps, centred)[:2]
        z = n if pre is None else n * pre
        en = en if pre is None else en * pre.abs() + E * z.abs()
        bz = en + u * (z.abs() + en) + t
    return h, eh + u * (h.abs() + eh) + t, z, bz


def _norm_back(a, g, eg, eps, centred):
    """(gradient of a, bound, n(a), bound) from n(a)'s gradient g, off by eg."""
    C = a.shape[1]
    n, en, r, rr = _norm(a, torch.zeros_like(a), eps, centred)
    both, gn = (g * n).mean(1, keepdim=True), (g.abs() + eg) * (n.abs() + en)
    eb = (eg * n.abs() + (g.abs() + eg) * en).mean(1, keepdim=True) + (C + 3) * E * gn.mean(1, keepdim=True)
    d, size = g - n * both, g.abs() + n.abs() * both.abs()
    ed = eg + n.abs() * eb + en * (both.abs() + eb)
    if centred:
        only = g.mean(1, keepdim=True)
        d, size = d - only, size + only.abs()
        ed = ed + eg.mean(1, keepdim=True) + (C + 3) * E * (g.abs() + eg).mean(1, keepdim=True)
    ed = ed + 4 * E * (size + ed)
    return d * r, (ed * r + d.abs() * r * rr) * (1 + rr) + 2 * E * (d * r).abs(), n, en


def norm_back(dh, dz, h, y, gate, post, pre, scale, eps, centred, norm_post, norm_pre, dtype):
    """[(dx, bound), (dy, bound), (dgate, bound), (dpost, bound), (dpre, bound)], None for what there is not."""
    T = h.shape[0]
    u, t = UNIT[dtype], TINY[dtype]
    total = lambda v, ev: (v.sum(0), ev.sum(0) + (T + 2) * E * (v.abs() + ev).sum(0))  # noqa: E731
    zero = torch.zeros_like(h)
    dx, ex, got = (zero if dh is None else dh), zero, {}
    if norm_pre:
        g = dz if pre is None else dz * pre
        d, ed, n, en = _norm_back(h, g, E * g.abs(), eps, centred)
        if pre is not None:
            got["pre"] = total(dz * n, dz.abs() * en + E * (dz * n).abs())
        dx = dx + d
        ex = ed + E * (dx.abs() + ed)
    got["x"] = dx, ex
    if y is not None:
        du, eu = scale * dx, abs(scale) * ex + E * (scale * dx).abs()
        v, ev, n, en = y, zero, None, None
        if norm_post:
            n, en = _norm(y, zero, eps, centred)[:2]
            v, ev = n, en
        if post is not None:
            v, ev = v * post, ev * post.abs() + E * (v * post).abs()
        if gate is not None:
            one = du * v, eu * (v.abs() + ev) + du.abs() * ev + 2 * E * (du * v).abs()
            got["gate"] = total(*one) if gate.dim() == 1 else one
            du, eu = du * gate, eu * gate.abs() + E * (du * gate).abs()
        if norm_post:
            if post is not None:
                got["post"] = total(du * n, eu * (n.abs() + en) + du.abs() * en + E * (du * n).abs())
            g, eg = (du, eu) if post is None else (du * post, eu * post.abs() + E * (du * post).abs())
            du, eu = _norm_back(y, g, eg, eps, centred)[:2]
        got["y"] = du, eu
    return [(got[k][0], got[k][1] + u * (got[k][0].abs() + got[k][1]) + t) if k in got else None for k in ("x", "y", "gate", "post", "pre")]
