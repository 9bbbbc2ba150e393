"""Arguments that calls of the binding may leave out, against a stand-in for the library."""
import pytest
import torch

from paper_1606_05688_amd import binding as B
from test_attention_devices import _Library
from test_block_host import F, _Shaped


def stand_in(monkeypatch):
    monkeypatch.setattr(B, "_lib", _Library())
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    _Library.called = False


def test_the_gradient_of_a_bias_takes_neither_inputs_nor_weights(monkeypatch):
    stand_in(monkeypatch)
    dout, z, db = _Shaped(0, (6, 8), F), _Shaped(0, (6, 8), F), _Shaped(0, (8,), F)
    ws = _Shaped(0, (1 << 20,), torch.uint8)
    assert B.znni_linear_backward(dout, None, None, z=z, act="gelu", inputs=False, weights=False, dbias=db, workspace=ws) == (None, None, db)
    assert _Library.called
