"""The layer of volume_block.py on a padded batch: rows behind the last sequence take no part in it and leave no trace in the weights' gradients."""
import pytest
import torch

from test_gpu_volume_layer import BOUND, _case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("rows", [1, 13, 300])
def test_rows_behind_the_last_sequence(dtype, rows):
    layer, lens, x, dout, pos, cu, window = _case(dtype)
    out, kept = layer.forward(x, pos, cu, max(lens), **window)
    dx, grads = layer.backward(dout, kept)
    T = x.shape[0]
    more = lambda t: torch.cat((t, torch.ones((rows, t.shape[1]), dtype=t.dtype, device="cuda")))  # noqa: E731
    x2, pos2, dout2 = more(x), more(pos), torch.cat((dout, torch.zeros((rows, dout.shape[1]), dtype=dtype, device="cuda")))
    for n in (4, 16, 64, 256, 1024):                               # memory that the calls' own tensors are made in
        held = [torch.full((n << 8,), float("nan"), device="cuda") for _ in range(32)]
        del held
    out2, kept2 = layer.forward(x2, pos2, cu, max(lens), **window)
    dx2, grads2 = layer.backward(dout2, kept2)
    assert all(torch.isfinite(t).all() for t in (out2, dx2, *grads2.values()))
    # sums over tokens may be taken in other parts: each within the layer's bound of the definition
    for name, a, b in (("out", out2[:T], out), ("dx", dx2[:T], dx), *((n, grads2[n], grads[n]) for n in grads)):
        off = (a.double() - b.double()).norm() / b.double().norm()
        assert off <= 2 * BOUND[dtype], (name, off)
    assert (dx2[T:] == 0).all()
