"""The block of volume_block.py: a whole volume against the definition in 64 bits, and the scan over the 8-bit cache against
the definition on what the cache holds after rounding, with pages that go back and come again."""
import numpy as np
import pytest
import torch

import attention_ref as R
from paper_1606_05688_amd.volume_block import VolumeBlock

pytestmark = pytest.mark.gpu


def _rounded(x, page_of, fills):
    """Values of the cache: codes under the scale of their page when it was last filled; `fills` are the token counts after each step."""
    pages = int(page_of[-1]) + 1
    ref = R.Cache(pages, x.shape[1], x.shape[2])
    table, have = np.arange(pages)[None], 0
    for n in fills:
        ref.append(x[have:n].double().cpu().numpy(), x[have:n].double().cpu().numpy(), table, [0, n - have], [have])
        have = n
        yield ref.tokens(0, table, n, 0)


@pytest.mark.parametrize("dtype,planes", [(torch.float32, 1), (torch.bfloat16, 2), (torch.float16, 3)])
def test_whole_and_scanned(dtype, planes):
    block = VolumeBlock(f=8, Hq=6, Hk=2, D=24, slabs=2, sinks=3, dtype=dtype)
    volume = torch.rand((1, 1, 11, 9, 10), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    q, k, v, plane = block.heads(volume)
    n = q.shape[0]
    r = R.rows(q.double().cpu(), k.double().cpu(), v.double().cpu(), torch.arange(n), 2 * plane, 0, 3, 24 ** -0.5)
    whole = block.whole(volume)
    R.check(whole, r[0], R.bound(dtype, *r))
    steps = list(block.scan(volume, planes))
    fills = [min(n, (i + 1) * planes * plane) for i in range(len(steps))]
    # the scan's own heads: the stem on fewer planes is the same layer up to fp32 rounding, so take them as they are
    ks, vs, qs = [], [], []
    for x0 in range(0, 9, planes):
        a = block.heads(volume[:, :, x0:min(9, x0 + planes) + 2].clone(), x0)
        qs.append(a[0]), ks.append(a[1]), vs.append(a[2])
    ks, vs = torch.cat(ks), torch.cat(vs)
    page_of = np.arange(n) // 64
    have = 0
    for got, a, kk, vv, m in zip(steps, qs, _rounded(ks, page_of, fills), _rounded(vs, page_of, fills), fills):
        r = R.rows(a.double().cpu(), kk, vv, torch.arange(have, m), 2 * plane, 0, 3, 24 ** -0.5)
        R.check(got, r[0], R.bound(dtype, *r), f"{have} .. {m}")
        have = m
    # and near the whole volume's: codes are within 2^-4 of their values
    parts = torch.cat(steps).float()
    assert (parts - whole.float()).norm() <= 2.0 ** -3 * whole.float().norm()
