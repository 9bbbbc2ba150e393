"""What is not finite in norms between blocks enters the results whose formulas it is in, and no others."""
import pytest
import torch

from paper_1606_05688_amd import binding as B
from test_gpu_block_norm import inputs

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gate", ["tokens", "shared", None])
@pytest.mark.parametrize("T,C", [(9, 72), (5, 600), (3, 3000), (2, 9000)])
def test_the_gradient_of_a_block_that_is_not_normed_does_not_depend_on_it(dtype, gate, T, C):
    """dy = scale dx gate, dx = dh + n'(h)[pre dz]: y is in neither; of the gate's gradient, scale dx y, it enters its own element."""
    i = inputs(T, C, dtype, gate, 30)
    i["post"] = None
    bad = i["y"].clone()
    where = [(0, 0, float("inf")), (T - 1, C - 1, float("nan")), (T // 2, C // 2, -float("inf"))]
    for t, c, value in where:
        bad[t, c] = value
    at = torch.isfinite(bad)
    for norm_pre in (True, False):
        kw = dict(gate=i["gate"], pre=i["pre"] if norm_pre else None, scale=0.7, norm_post=False, norm_pre=norm_pre)
        dz = i["dz"] if norm_pre else None
        plain = B.znni_block_norm_backward(i["dh"], dz, i["x"], i["y"], **kw)
        got = B.znni_block_norm_backward(i["dh"], dz, i["x"], bad, **kw)
        for n in (0, 1, 4):
            assert (got[n] is None) == (plain[n] is None) and (got[n] is None or torch.equal(got[n], plain[n]))
        if gate == "tokens":
            assert torch.equal(got[2][at], plain[2][at]) and not torch.isfinite(got[2][~at]).any()
        elif gate == "shared":
            assert torch.equal(got[2][at.all(0)], plain[2][at.all(0)]) and not torch.isfinite(got[2][~at.all(0)]).any()
