"""Windowed attention where values are infinite or enormous under weights that vanish."""
import pytest
import torch

import attention_ref as R
from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
CALLS = [(1, 1, 200), (1, 40, 300), (1, 1, 5000), (410, 3, 200), (1, 33, 2500), (1, 300, 1500), (1, 2, 1100), (30, 40, 300), (410, 40, 300)]


def _case(dtype, nq, nk, D, spread):
    """Keys whose scores climb by `spread` from the first to the last."""
    g = torch.Generator().manual_seed(nq + nk + D)
    q, k = torch.zeros(nq, 2, D), torch.zeros(nk, 1, D)
    q[..., 0], k[..., 0] = 1.0, (torch.arange(nk) * (spread / nk)).round().unsqueeze(-1)
    v = torch.randn(nk, 1, D, generator=g)
    return q.to(dtype), k.to(dtype), v.to(dtype)


def _check(dtype, q, k, v, copies, left, sinks):
    nq, nk = q.shape[0], k.shape[0]
    ref = R.rows(q.double(), k.double(), v.double(), torch.arange(nq) + nk - nq, left, 0, sinks, 1.0)
    cu = [torch.arange(copies + 1, dtype=torch.int32, device=DEV) * n for n in (nq, nk)]
    got = B.znni_attn_window(*(x.repeat(copies, 1, 1).to(DEV) for x in (q, k, v)), *cu, nq, nk, left=left, sinks=sinks,
                             scale=1.0).view(copies, *q.shape)
    fine = torch.isfinite(ref[0])
    R.check(got[0], ref[0], torch.where(fine, R.bound(dtype, *ref), torch.ones_like(ref[0])), f"{left} {sinks}")
    assert torch.equal(torch.nan_to_num(got, nan=-7.0), torch.nan_to_num(got[:1], nan=-7.0).expand_as(got))
    return ref[0]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [64, 40, 128, 96, 24])
@pytest.mark.parametrize("copies,nq,nk", CALLS)
def test_infinities_under_weights_that_vanish(dtype, D, copies, nq, nk):
    """A row that sees an infinity has it, however small its weight (e^-190 and less here) and however the keys are shared out."""
    print(f"[infinities] {dtype} {D} {copies} {nq} {nk}", flush=True)
    q, k, v = _case(dtype, nq, nk, D, 200)
    v[1, 0, 0], v[2, 0, 5], v[nk // 2, 0, D - 1] = float("inf"), float("-inf"), float("inf")
    v[3, 0, 7], v[nk // 3, 0, 7] = float("inf"), float("-inf")          # both: no number
    v[4, 0, 9] = float("nan")
    v[nk - 1, 0, 3] = float("-inf")                                     # and one under the largest weight of the last row
    for left, sinks in ((B.ALL, 0), (nk // 2 + 3, 2), (20, 4)):
        out = _check(dtype, q, k, v, copies, left, sinks)
        assert torch.isinf(out).any() and torch.isfinite(out).any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 40])
@pytest.mark.parametrize("copies,nq,nk", CALLS)
def test_enormous_values_under_weights_that_vanish(dtype, D, copies, nq, nk):
    """1e37 under a weight of e^-190 is nothing."""
    q, k, v = _case(dtype, nq, nk, D, 200)
    k[40:64] = 0                                                        # (the second half of the first tile, too)
    v[:5], v[40:50] = 1e37, -2e37
    for left, sinks in ((B.ALL, 0), (20, 4)):
        _check(dtype, q, k, v, copies, left, sinks)
