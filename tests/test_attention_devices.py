"""Arguments of the attention calls on another GPU than the first tensor's are refused before the library is called."""
import pytest
import torch

from paper_1606_05688_amd import binding as B
from test_attention_streams import _Tensor


class _On(_Tensor):
    def __init__(self, gpu, shape, dtype):
        super().__init__(shape, dtype)
        self.gpu, self.device = gpu, torch.device("cuda", gpu)

    def get_device(self):
        return self.gpu


class _Library:
    called = False

    def __getattr__(self, name):
        def call(*args):
            if not name.endswith("workspace"):
                _Library.called = True
            return 0
        return call


F, I, U, X = torch.float16, torch.int32, torch.uint8, torch.float32
CALLS = {
    "rope": (lambda a: B.znni_rope_axes(a["q"], a["k"], a["pos"], a["freq"], (4, 4), out_q=a["oq"], out_k=a["ok"]),
             dict(q=((6, 4, 32), F), k=((6, 2, 32), F), pos=((6, 2), I), freq=((8,), X), oq=((6, 4, 32), F), ok=((6, 2, 32), F))),
    "window": (lambda a: B.znni_attn_window(a["q"], a["k"], a["v"], a["cu_q"], a["cu_k"], 6, 9, out=a["out"], workspace=a["ws"]),
               dict(q=((6, 4, 32), F), k=((9, 2, 32), F), v=((9, 2, 32), F), cu_q=((2,), I), cu_k=((2,), I), out=((6, 4, 32), F), ws=((256,), U))),
    "append": (lambda a: B.znni_kv8_append(a["kc"], a["vc"], a["sc"], a["k"], a["v"], a["table"], a["cu"], a["start"], 9),
               dict(k=((9, 2, 32), F), v=((9, 2, 32), F), kc=((3, 2, 64, 32), U), vc=((3, 2, 32, 64), U), sc=((3, 2, 2), X),
                    table=((1, 3), I), cu=((2,), I), start=((1,), I))),
    "cache": (lambda a: B.znni_kv8_attn(a["q"], a["kc"], a["vc"], a["sc"], a["table"], a["lens"], 99, out=a["out"], workspace=a["ws"]),
              dict(q=((1, 2, 4, 32), F), kc=((3, 2, 64, 32), U), vc=((3, 2, 32, 64), U), sc=((3, 2, 2), X), table=((1, 3), I), lens=((1,), I),
                   out=((1, 2, 4, 32), F), ws=((256,), U))),
}
FIRST = {"rope": "q", "window": "q", "append": "k", "cache": "q"}


def _call(monkeypatch, name, elsewhere=None):
    monkeypatch.setattr(B, "_lib", _Library())
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    _Library.called = False
    call, args = CALLS[name]
    call({n: _On(1 if n == elsewhere else 0, *a) for n, a in args.items()})


@pytest.mark.parametrize("name", CALLS)
def test_all_on_one_gpu(monkeypatch, name):
    _call(monkeypatch, name)
    assert _Library.called


@pytest.mark.parametrize("name,argument", [(n, a) for n, (_, args) in CALLS.items() for a in args if a != FIRST[n]])
def test_one_on_another_gpu(monkeypatch, name, argument):
    with pytest.raises(AssertionError):
        _call(monkeypatch, name, argument)
    assert not _Library.called
