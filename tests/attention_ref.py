"""The attention operators' definitions in 64 bits on the CPU, row by row where a mask decides what is touched, and bounds
on what rounding may do to a kernel that follows them in 32 bits."""
import numpy as np
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
PAGE = 64


def rope(x, pos, freq, sections, pairing):
    """x [T, H, D] float64, pos [T, axes], freq [R] -> turned."""
    R = sum(sections)
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = pos.double()[:, axis] * freq.double()
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    y = x.clone()
    u, v = (slice(0, R), slice(R, 2 * R)) if pairing == "halves" else (slice(0, 2 * R, 2), slice(1, 2 * R, 2))
    y[..., u] = x[..., u] * c - x[..., v] * s
    y[..., v] = x[..., u] * s + x[..., v] * c
    return y


def visible(p, n, left, right, sinks):
    """Keys below n that a row at position p sees."""
    j = torch.arange(n)
    return j[(j <= p + right) & ((j >= p - left) | (j < sinks))]


def rows(q, k, v, positions, left, right, sinks, scale):
    """q [n, H, D], k and v [m, Hk, D] float64; row i at positions[i].  Only what a row sees is touched.
    Returns (out, sum of weights times |v|, bound on the error of a score in fp32, largest |v| seen of each element, keys seen)."""
    n, H, D = q.shape
    G = H // k.shape[1]
    out, mass = torch.zeros_like(q), torch.zeros_like(q)
    ds, vmax, count = torch.zeros(n, H, 1).double(), torch.zeros_like(q), torch.zeros(n, 1, 1).double()
    for i in range(n):
        see = visible(int(positions[i]), k.shape[0], left, right, sinks)
        if not len(see):
            continue
        kk, vv = k[see].repeat_interleave(G, 1), v[see].repeat_interleave(G, 1)          # [m, H, D]
        s = (q[i] * kk).sum(-1) * scale                                                  # [m, H]
        w = torch.exp(s - s.max(0).values)
        w = w / w.sum(0)
        out[i] = (w[..., None] * vv).sum(0)
        mass[i] = (w[..., None] * vv.abs()).sum(0)
        size = (q[i].abs() * kk.abs()).sum(-1).max(0).values * abs(scale)
        ds[i, :, 0] = (D + 8) * 2.0 ** -24 * size + 2.0 ** -22 * s.abs().max(0).values
        vmax[i] = vv.abs().amax(0)
        count[i] = len(see)
    return out, mass, ds, vmax, count


def bound(dtype, out, mass, ds, vmax, count):
    """Scores off by ds move each weight by 2 ds, sums of `count` terms lose count * 2^-24, weights are rounded to the type (below
    its normal range by 2^-25 at most) before they meet the values, the result once more."""
    u = UNIT[dtype]
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    return u * out.abs() + (u + 2 * ds + (count + 16) * 2.0 ** -23) * mass * 1.01 + tiny * (count * vmax + 1) + 1e-37


def check(got, exp, tol, what=""):
    got, exp = got.double().cpu(), exp.double()
    assert torch.equal(torch.isnan(got), torch.isnan(exp)), f"{what}: NaN elsewhere"
    inf = torch.isinf(exp)
    assert torch.equal(got[inf], exp[inf]) and not torch.isinf(got[~inf]).any(), f"{what}: infinities elsewhere"
    fine = torch.isfinite(exp)
    over = ((got - exp).abs()[fine] / tol[fine])
    assert over.numel() == 0 or over.max() <= 1, f"{what}: {over.max():.3g} times the bound"


# ---- the 8-bit cache ----------------------------------------------------------------------------------------------

def e4m3(code):
    """Value of codes (uint8 tensor): 4 exponent bits of bias 7, 3 mantissa bits, no infinity, NaN = all ones."""
    c = code.to(torch.int64)
    e, m = (c >> 3) & 15, c & 7
    v = torch.where(e == 0, m.double() * 2.0 ** -9, (8 + m).double() * torch.exp2(e.double() - 10))
    v = torch.where((e == 15) & (m == 7), torch.full_like(v, float("nan")), v)
    return torch.where(c >= 128, -v, v)


_VALUES = e4m3(torch.arange(127, dtype=torch.uint8)).numpy()            # 0 .. 448, rising


def to_e4m3(y):
    """Nearest value, ties to the even code, infinities and what is over 448 to 448, NaN stay; as values."""
    y = np.asarray(y, dtype=np.float64)
    a = np.minimum(np.abs(y), 448.0)
    hi = np.clip(np.searchsorted(_VALUES, np.nan_to_num(a)), 1, 126)
    lo = hi - 1
    dl, dh = a - _VALUES[lo], _VALUES[hi] - a
    pick = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(y), np.nan, np.copysign(_VALUES[pick], y))


class Cache:
    """Values and exponents of a cache, by the definition of its filling."""

    def __init__(self, pages, Hk, D):
        self.k = np.zeros((pages, Hk, PAGE, D))
        self.v = np.zeros((pages, Hk, PAGE, D))
        self.e = np.full((pages, Hk, 2), -126)

    def append(self, k, v, table, cu, start):
        for b in range(len(start)):
            n, at = int(cu[b + 1] - cu[b]), int(start[b])
            done = 0
            while done < n:
                i, slot = divmod(at + done, PAGE)
                m = min(n - done, PAGE - slot)
                page = int(table[b, i]) if i < table.shape[1] else -1
                t = slice(int(cu[b]) + done, int(cu[b]) + done + m)
                if 0 <= page < len(self.k):
                    for which, (pool, x) in enumerate(((self.k, k), (self.v, v))):
                        for h in range(x.shape[1]):
                            new = x[t, h].astype(np.float64)
                            fin = np.abs(new[np.isfinite(new)])
                            top = fin.max() if fin.size else 0.0
                            e = -126
                            while top > 448 * 2.0 ** e:
                                e += 1
                            old = self.e[page, h, which]
                            if slot and old >= e:
                                e = old
                            elif slot:
                                pool[page, h, :slot] = to_e4m3(pool[page, h, :slot] * 2.0 ** float(old - e))
                            pool[page, h, slot:slot + m] = to_e4m3(new * 2.0 ** float(-e))
                            self.e[page, h, which] = e
                done += m

    def tokens(self, b, table, n, which):
        """[n, Hk, D] values of sequence b."""
        pool = self.v if which else self.k
        x = [pool[int(p)] * 2.0 ** self.e[int(p), :, which, None, None].astype(np.float64) for p in table[b, :-(-n // PAGE)]]
        return torch.from_numpy(np.concatenate(x, 1)[:, :n].transpose(1, 0, 2).copy()) if x else None
