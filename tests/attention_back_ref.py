"""Gradients of windowed attention in 64 bits on the CPU with bounds on what rounding may do to a kernel that works weights out again from
32-bit statistics, rounds weights and their gradients to the type before the last products, and each result once."""
import torch

from attention_ref import UNIT, check  # noqa: F401

E = 2.0 ** -24


def seen(nq, nk, left, right, sinks):
    p, j = torch.arange(nq)[:, None] + (nk - nq), torch.arange(nk)[None, :]
    return (j <= p + right) & ((j >= p - left) | (j < sinks))


def forward(q, k, v, left, right, sinks, scale):
    """q [nq, Hq, D], k, v [nk, Hk, D] float64 -> (out, sum of exp(scores - largest), largest score) of each row and head."""
    nq, Hq, _ = q.shape
    nk, Hk, _ = k.shape
    out, total, top = torch.zeros_like(q), torch.zeros(nq, Hq).double(), torch.zeros(nq, Hq).double()
    see = seen(nq, nk, left, right, sinks)
    for h in range(Hq if nk else 0):
        s = torch.where(see, scale * q[:, h] @ k[:, h * Hk // Hq].T, -torch.inf)
        m = s.max(1).values
        m = torch.where(torch.isinf(m), 0.0, m)
        w = torch.exp(s - m[:, None])
        top[:, h], total[:, h] = m, w.sum(1)
        out[:, h] = torch.where(total[:, h, None] > 0, w @ v[:, h * Hk // Hq] / total[:, h, None], 0.0)
    return out, total, top


def backward(q, k, v, dout, left, right, sinks, scale, dtype):
    """[(dq, bound), (dk, bound), (dv, bound)] of one sequence."""
    (nq, Hq, D), (nk, Hk, _) = q.shape, k.shape
    u, f16 = UNIT[dtype], dtype == torch.float16
    if nq == 0 or nk == 0:
        return [(torch.zeros_like(x), torch.full_like(x, 1e-37)) for x in (q, k, v)]
    got = [(torch.zeros_like(x), torch.zeros_like(x)) for x in (q, k, v)]
    see = seen(nq, nk, left, right, sinks)
    count = see.sum(1)
    # fp16: half the least step, after weights were taken times 2^15 and their gradients to a largest of 2^13
    tiny_p = 2.0 ** -40 if f16 else 0.0
    peak = D * dout.abs().max() * v.abs().max()
    tiny_s = 2.0 ** -38 * peak if f16 else 0.0
    r = u if dtype != torch.float32 else 0.0
    for h in range(Hq):
        a, b, c, d = q[:, h], k[:, h * Hk // Hq], v[:, h * Hk // Hq], dout[:, h]
        s = torch.where(see, scale * a @ b.T, -torch.inf)
        p = torch.where(see, torch.exp(s - torch.logsumexp(s, 1, keepdim=True)), 0.0)
        size = torch.where(see, abs(scale) * a.abs() @ b.abs().T, 0.0).amax(1)
        ds = (D + 8) * E * size + 4 * E * torch.where(see, s.abs(), 0.0).amax(1)     # a score, and the reference, are off by this
        rp = (2 * (ds + ds) + (count + 24) * 2 * E)[:, None]                          # a weight relative to itself: scores here and in the sum
        dp = d @ c.T
        delta = (p * dp).sum(1, keepdim=True)
        out = p @ c
        eo = u * out.abs() + (r + rp) * (p @ c.abs()) * 1.01 + (2.0 ** -25 if f16 else 0.0) * (1 + count[:, None] * c.abs().max())
        ed = (d.abs() * eo).sum(1, keepdim=True) + (D + 4) * E * (d.abs() * out.abs()).sum(1, keepdim=True)
        ep = (D + 6) * E * (d.abs() @ c.abs().T)
        g = p * (dp - delta)
        eg = p * (rp * (dp - delta).abs() + (ep + ed + 4 * E * (dp.abs() + delta.abs())) * (1 + rp))
        eg = eg + r * (g.abs() + eg) + tiny_s * see
        for (y, by), x, w, ew, f in ((got[0], b, g, eg, scale), (got[1], a, g.T, eg.T, scale), (got[2], d, p.T, (p * (rp + r + rp * r) + tiny_p * see).T, 1.0)):
            head = h if y is got[0][0] else h * Hk // Hq
            y[:, head] += f * (w @ x)
            by[:, head] += abs(f) * (ew @ x.abs() + (w.shape[1] * (Hq // Hk) + 4) * E * ((w.abs() + ew) @ x.abs()))
    return [(y, by + u * (y.abs() + by) + (2.0 ** -25 if f16 else 1e-37)) for y, by in got]
