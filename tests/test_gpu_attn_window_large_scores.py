"""Windowed attention where scores are large and exact, and only their small differences count."""
import pytest
import torch

import attention_ref as R
from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
FACTORS = (256.0, 1.0, 1.0, 1.0)


def _terms(score, dtype):
    """[n, 4] of the type whose products with FACTORS sum to the scores, which are exact: every partial sum is, too."""
    rest, out = score.double().clone(), []
    for f in FACTORS:
        x = (rest / f).float()
        t = x.to(dtype)
        over = t.double().abs() > x.double().abs()
        t = torch.where(over, torch.nextafter(t.float(), torch.zeros_like(x)).to(dtype), t)
        if dtype != torch.float32:              # towards zero in the type: one of its values below
            bits = x.view(torch.int32)
            cut = 16 if dtype == torch.bfloat16 else 13
            t = (bits >> cut << cut).view(torch.float32).to(dtype)
        out.append(t)
        rest = rest - t.double() * f
    assert (rest == 0).all()
    return torch.stack(out, -1)


# scale, score that all lie near, step of the scores: (scale * score * log2 e is 2.9e6; 9.2e7; on both sides of 2^26)
LEVELS = [(0.125, 16.0e6, 1.0), (0.125, -16.0e6, 1.0), (8.0, 8.0e6, 0.5), (8.0, 5814532.0, 0.5)]
# steps above the level of each key's score; with a scale of 8 a step is four powers of e, and there are fewer of them
SHAPES = {
    "two halves of a tile": lambda j, few: torch.where(j % 64 < 32, 0, 1 if few else 4) + (0 if few else j % 3),
    "rising": lambda j, few: (j // 64).clamp(max=3) if few else j // 64 * 13 + j % 5,
    "falling": lambda j, few: -(j // 64).clamp(max=3) if few else -(j // 64 * 13) + j % 5,
    "late": lambda j, few: torch.where(j == j.max(), 1 if few else 12, 0 if few else j % 2),
    "tile by tile": lambda j, few: j // 64 % 2 * (1 if few else 9),
    "part by part": lambda j, few: j // 600 % 2 * (1 if few else 9),
}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("level", LEVELS, ids=lambda x: f"{x[0]}-{x[1]:g}")
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("copies,nq,nk", [(1, 1, 200), (1, 40, 300), (1, 1, 5000), (410, 3, 200), (1, 33, 2500), (30, 40, 300), (410, 40, 300)])
def test_differences_of_large_scores(dtype, level, shape, copies, nq, nk):
    """Rows in one wave and shared by several, keys whole and split, maxima that move from tile to tile."""
    scale, base, step = level
    D = 64
    print(f"[large scores] {dtype} {level} {shape} {copies} {nq} {nk}", flush=True)
    score = base + step * SHAPES[shape](torch.arange(nk), scale == 8.0).double()
    k = torch.zeros(nk, 1, D)
    k[:, 0, :4] = _terms(score, dtype).float()
    q = torch.zeros(nq, 1, D)
    q[:, 0, :4] = torch.tensor(FACTORS)
    v = torch.randn(nk, 1, D, generator=torch.Generator().manual_seed(nk))
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    out, mass, _, vmax, count = R.rows(q.double(), k.double(), v.double(), torch.arange(nq) + nk - nq, B.ALL, 0, 0, scale)
    # scores are exact, so what is left is what follows them: exponents up to 16, each worked out in up to four roundings of 2^-24
    ds = torch.full_like(out[..., :1], 4 * 16 * 2.0 ** -24)
    cu = [torch.arange(copies + 1, dtype=torch.int32, device=DEV) * n for n in (nq, nk)]
    got = B.znni_attn_window(*(x.repeat(copies, 1, 1).to(DEV) for x in (q, k, v)), *cu, nq, nk, scale=scale).view(copies, nq, 1, D)
    assert torch.equal(got, got[:1].expand_as(got))
    R.check(got[0], out, R.bound(dtype, out, mass, ds, vmax, count))
