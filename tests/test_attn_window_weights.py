"""How many bits of a weight windowed attention keeps where a sequence has few rows: sequences of three keys, whose scores are
exact, so that the weights' own rounding is what is left; results of all sizes, down to those that nearly cancel."""
import pytest
import torch

import attention_ref as R
from paper_1606_05688_amd import binding as B

DEV = "cuda:0"
HQ, HK, D, SCALE = 4, 2, 64, 0.9
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _inputs(dtype, n):
    """q [n, HQ, D], k and v [n * 3, HK, D], values with so few bits that every product with a query is exact."""
    g = torch.Generator().manual_seed(4)
    q = torch.zeros(n, HQ, D)
    q[..., 0] = 1 + torch.randint(0, 128, (n, HQ), generator=g) / 128.0
    k = torch.randint(-7, 8, (n * 3, HK, D), generator=g) / 4.0
    v = torch.randint(8, 16, (n * 3, HK, D), generator=g) * torch.exp2(-torch.randint(0, 4, (n * 3, HK, D), generator=g).float())
    v *= 1.0 - 2.0 * torch.randint(0, 2, v.shape, generator=g)
    return q.to(dtype), k.to(dtype), v.to(dtype)


def _exact(q, k, v):
    """(results, sums of weights times |v|, weights over the largest [n, HQ, 3], values [n, HQ, 3, D]) in 64 bits."""
    G = HQ // HK
    kk, vv = (x.double().view(-1, 3, HK, D).permute(0, 2, 1, 3).repeat_interleave(G, 1) for x in (k, v))
    s = (q[:, :, None].double() * kk).sum(-1) * SCALE
    p = torch.exp(s - s.amax(-1, keepdim=True))
    total = p.sum(-1, keepdim=True)
    return (p[..., None] * vv).sum(2) / total, (p[..., None] * vv.abs()).sum(2) / total, p, vv


def _bound(dtype, out, mass):
    """In units of 2^-24: scores up to 1.75 * 2 * 0.9 * log2 e = 4.6 powers of two, each worked out in at most four roundings, their
    difference in one more, the power in two: (8 * 4.6 + 9.2) ln 2 + 2 < 38.8 of a weight at most, and as much of their sum; sums and
    the quotient 12; the weight's own rounding, 16 bits in 16-bit types, none in fp32; the result's."""
    own = 0.0 if dtype == torch.float32 else 2.0 ** -16
    return R.UNIT[dtype] * out.abs() + (own + (2 * 38.8 + 12) * 2.0 ** -24) * mass


@pytest.mark.parametrize("dtype", TYPES[1:])
def test_the_bound_tells_weights_of_one_value(dtype):
    out, mass, p, vv = _exact(*_inputs(dtype, 256))
    one = p.to(dtype).double()
    worst = [((((w[..., None] * vv).sum(2) / p.sum(-1, keepdim=True)).to(dtype).double() - out).abs() / _bound(dtype, out, mass)).max().item()
             for w in (one, one + (p - one).to(dtype).double())]
    assert worst[1] <= 1 < 2 < worst[0], worst


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 8, 150, 1000])
@pytest.mark.parametrize("max_q", [1, 32])
def test_bits_of_a_weight(dtype, n, max_q):
    """Single sequences and so many that all compute units have some; any bound on the rows that still leaves few."""
    q, k, v = _inputs(dtype, n)
    cu = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    got = B.znni_attn_window(q.to(DEV), k.to(DEV), v.to(DEV), cu, 3 * cu, max_q, 3, scale=SCALE)
    out, mass, _, _ = _exact(q, k, v)
    R.check(got, out, _bound(dtype, out, mass))
