"""Gradients of products of which only some are wanted, or none."""
import pytest
import torch

from paper_1606_05688_amd import binding as B
from test_gpu_linear import inputs

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", [None, "relu", "gelu", "silu"])
def test_none_wanted(dtype, act):
    """Nothing is written: not the workspace that the caller passes, nor any input."""
    x, w, _, z, dout = inputs(70, 136, 72, dtype, 20)
    ws = torch.full((1 << 16,), 77, dtype=torch.uint8, device="cuda")
    kept = [t.clone() for t in (x, w, z, dout)]
    kw = dict(z=None if act is None else z, act=act, inputs=False, weights=False, bias=False)
    assert B.znni_linear_backward(dout, x, w, **kw) == (None, None, None)
    assert B.znni_linear_backward(dout, x, w, workspace=ws, **kw) == (None, None, None)
    torch.cuda.synchronize()
    assert (ws == 77).all() and all(torch.equal(a, b) for a, b in zip(kept, (x, w, z, dout)))
