"""Windowed attention with scales that are negative, zero or next to it."""
import pytest
import torch

import attention_ref as R
from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
CALLS = [(1, 1, 200), (1, 40, 300), (1, 1, 5000), (210, 5, 70), (1, 33, 2500), (30, 40, 300), (410, 40, 300)]


def _check(dtype, q, k, v, copies, left, sinks, scale, ds=None):
    nq, nk = q.shape[0], k.shape[0]
    ref = list(R.rows(q.double(), k.double(), v.double(), torch.arange(nq) + nk - nq, left, 0, sinks, scale))
    if ds is not None:
        ref[2] = torch.full_like(ref[2], ds)
    cu = [torch.arange(copies + 1, dtype=torch.int32, device=DEV) * n for n in (nq, nk)]
    got = B.znni_attn_window(*(x.repeat(copies, 1, 1).to(DEV) for x in (q, k, v)), *cu, nq, nk, left=left, sinks=sinks,
                             scale=scale).view(copies, *q.shape)
    assert torch.equal(got, got[:1].expand_as(got))
    R.check(got[0], ref[0], R.bound(dtype, *ref), f"{scale}")


def _inputs(dtype, nq, nk, Hq, Hk, D):
    g = torch.Generator().manual_seed(nq + nk)
    return tuple(torch.randn(n, h, D, generator=g).to(dtype) for n, h in ((nq, Hq), (nk, Hk), (nk, Hk)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("copies,nq,nk", CALLS)
@pytest.mark.parametrize("scale", [-0.3, -2.0, 0.0, -0.0, 1e-30, 1e-38, -1e-39, 1e-42, 1.5e-45])
def test_any_scale(dtype, copies, nq, nk, scale):
    print(f"[scale] {dtype} {scale} {copies} {nq} {nk}", flush=True)
    q, k, v = _inputs(dtype, nq, nk, 2, 1, 64)
    for left, sinks in ((B.ALL, 0), (50, 3)):
        _check(dtype, q, k, v, copies, left, sinks, scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("copies,nq,nk", CALLS)
@pytest.mark.parametrize("scale", [0.0, 1e-40, -1e-40])
def test_no_scale_and_enormous_scores(dtype, copies, nq, nk, scale):
    """Scores of 2^124: a scale of zero makes them equal all the same, one of 1e-40 takes them to 2e-3."""
    q, k, v = _inputs(dtype, nq, nk, 2, 1, 64)
    q, k = q.sign() * 2.0 ** 60, k.sign() * 2.0 ** 58
    # sums of +-2^118 are exact; a scale below the normal range has 16 bits, of the scaled score 64 * 2^118 * 1e-40 at most
    _check(dtype, q, k, v, copies, 50, 3, scale, ds=64 * 2.0 ** 118 * 1e-40 * 2.0 ** -15 + 2.0 ** -22)
