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


@pytest.mark.parametrize("dtype", TYPES)
def test_the_bias_alone(dtype):
    x, w, _, z, dout = inputs(70, 136, 72, dtype, 21)
    for act in (None, "silu"):
        kw = dict(z=None if act is None else z, act=act)
        whole = B.znni_linear_backward(dout, x, w, **kw)
        got = B.znni_linear_backward(dout, None, None, inputs=False, weights=False, **kw)
        assert got[0] is None and got[1] is None and torch.equal(got[2], whole[2])
        # and each product without the operand that only the other takes
        dx, dw, _ = B.znni_linear_backward(dout, None, w, weights=False, bias=False, **kw)
        assert dw is None and torch.equal(dx, whole[0])
        dx, dw, _ = B.znni_linear_backward(dout, x, None, inputs=False, bias=False, **kw)
        assert dx is None and torch.equal(dw, whole[1])


def test_operands_that_are_missing_are_refused():
    x, w, _, _, dout = inputs(8, 16, 24, torch.bfloat16, 22)
    for a, b in ((None, w), (x, None), (None, None)):
        with pytest.raises(RuntimeError):
            B.znni_linear_backward(dout, a, b)
