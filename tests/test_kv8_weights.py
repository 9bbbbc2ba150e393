"""How many bits of a weight the attention over the 8-bit cache keeps: sequences of three tokens, whose scores are exact, so that
the weights' own rounding is what is left; results of all sizes, down to those that nearly cancel."""
import pytest
import torch

import attention_ref as R
from paper_1606_05688_amd import binding as B

DEV = "cuda:0"
BN, HQ, HK, D, SCALE = 256, 4, 2, 64, 0.9
TERMS = {torch.float32: 3, torch.bfloat16: 2, torch.float16: 2}         # of 8 bits: 24 bits of a weight in fp32, 16 in 16-bit types


def _inputs(dtype):
    """q [BN, 1, HQ, D], k and v [BN * 3, HK, D]: every value has a code, every product with a query is exact."""
    g = torch.Generator().manual_seed(4)
    q = torch.zeros(BN, 1, HQ, D)
    q[..., 0] = 1 + torch.randint(0, 128, (BN, 1, HQ), generator=g) / 128.0
    k = torch.randint(-7, 8, (BN * 3, HK, D), generator=g) / 4.0
    v = torch.randint(8, 16, (BN * 3, HK, D), generator=g) * torch.exp2(-torch.randint(0, 4, (BN * 3, HK, D), generator=g).float())
    v *= 1.0 - 2.0 * torch.randint(0, 2, v.shape, generator=g)
    return q.to(dtype), k.to(dtype), v.to(dtype)


def _exact(q, k, v):
    """(results [BN, HQ, D], sums of weights times |v|, weights over the largest [BN, HQ, 3], values [BN, HQ, 3, D]) in 64 bits."""
    G = HQ // HK
    kk, vv = (x.double().view(BN, 3, HK, D).permute(0, 2, 1, 3).repeat_interleave(G, 1) for x in (k, v))
    s = (q[:, 0, :, None].double() * kk).sum(-1) * SCALE
    p = torch.exp(s - s.amax(-1, keepdim=True))
    total = p.sum(-1, keepdim=True)
    return (p[..., None] * vv).sum(2) / total, (p[..., None] * vv.abs()).sum(2) / total, p, vv


def _bound(dtype, out, mass):
    """In units of 2^-24: scores up to 1.75 * 2 * 0.9 * log2 e = 4.6 powers of two, each worked out in four roundings, their difference in
    one more, the power in two: (8 * 4.6 + 9.2) ln 2 + 2 < 38.8 of a weight at most, and as much of their sum; sums and the quotient
    12; the weight's own rounding, 2^-16 or 2^-24; the result's."""
    own = 2.0 ** (-8 * TERMS[dtype])
    return R.UNIT[dtype] * out.abs() + (own + (2 * 38.8 + 12) * 2.0 ** -24) * mass


def _rounded(p, terms):
    """p as a sum of so many bf16, all but the last cut off."""
    rest, got = p.float(), torch.zeros_like(p)
    for n in range(terms):
        t = rest.bfloat16().float() if n == terms - 1 else (rest.view(torch.int32) >> 16 << 16).view(torch.float32)
        got += t.double()
        rest = rest - t
    return got


@pytest.mark.parametrize("dtype", TERMS)
def test_the_bound_tells_one_term_fewer(dtype):
    out, mass, p, vv = _exact(*_inputs(dtype))
    worst = {}
    for terms in (TERMS[dtype], TERMS[dtype] - 1):
        got = ((_rounded(p, terms)[..., None] * vv).sum(2) / p.sum(-1, keepdim=True)).to(dtype).double()
        worst[terms] = ((got - out).abs() / _bound(dtype, out, mass)).max().item()
    assert worst[TERMS[dtype]] <= 1 < 2 < worst[TERMS[dtype] - 1], worst


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TERMS)
def test_bits_of_a_weight(dtype):
    q, k, v = _inputs(dtype)
    pools = B.kv8_alloc(BN, HK, D, DEV)
    table = torch.arange(BN, dtype=torch.int32, device=DEV)[:, None]
    cu = 3 * torch.arange(BN + 1, dtype=torch.int32, device=DEV)
    zero = torch.zeros(BN, dtype=torch.int32, device=DEV)
    B.znni_kv8_append(*pools, k.to(DEV), v.to(DEV), table, cu, zero, 3)
    kc, vc, sc = (x.cpu() for x in pools)
    held = [(R.e4m3(kc) * sc[:, :, 0, None, None]).permute(0, 2, 1, 3)[:, :3], (R.e4m3(vc) * sc[:, :, 1, None, None]).permute(0, 3, 1, 2)[:, :3]]
    assert torch.equal(held[0].reshape(-1, HK, D), k.double()) and torch.equal(held[1].reshape(-1, HK, D), v.double())
    out, mass, _, _ = _exact(q, k, v)
    got = B.znni_kv8_attn(q.to(DEV), *pools, table, zero + 3, 3, scale=SCALE)
    R.check(got[:, 0], out, _bound(dtype, out, mass))
