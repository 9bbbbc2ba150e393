"""Calls on a stream that is not torch's current one: what a call copies and allocates is ordered with what it launches."""
import contextlib

import pytest
import torch

from paper_1606_05688_amd import binding as B

DEV = "cuda:0"


class _Tensor:
    """What the binding asks of a tensor on a GPU, without one.  Copies note the stream that they run on."""
    is_cuda = True
    device = torch.device(DEV)

    def __init__(self, shape, dtype, strides=None, log=None, current=None):
        self.shape, self.dtype, self.log, self.current = torch.Size(shape), dtype, log, current
        self.strides = strides or torch.empty(shape, device="meta").stride()

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def get_device(self):
        return 0

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 0x1000

    def is_contiguous(self):
        return tuple(self.strides) == tuple(torch.empty(self.shape, device="meta").stride())

    def contiguous(self):
        self.log.append(("copy", self.current[-1]))
        return _Tensor(self.shape, self.dtype, None, self.log, self.current)

    def record_stream(self, stream):
        pass


class _Library:
    def __init__(self, log):
        self.log = log

    def znni_kv8_attn_workspace(self, *args):
        return 0

    def znni_kv8_attn(self, *args):
        self.log.append(("launch", args[-1]))
        return 0


class _Stream:
    device = torch.device(DEV)

    def __init__(self, address):
        self.cuda_stream = address


def test_a_copy_of_the_queries_runs_on_the_stream_of_the_launch(monkeypatch):
    main, side = _Stream(0), _Stream(77)
    log, current = [], [main.cuda_stream]

    @contextlib.contextmanager
    def switched(stream):
        current.append(stream.cuda_stream)
        yield
        current.pop()

    monkeypatch.setattr(torch.cuda, "stream", switched)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: main)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: current[-1], raising=False)
    monkeypatch.setattr(B, "_lib", _Library(log))
    Bn, Lq, Hq, Hk, D = 3, 2, 4, 2, 32
    q = _Tensor((Bn, Lq, Hq, D), torch.float16, (Hq * D, Bn * Hq * D, D, 1), log, current)          # [Lq, B, ..] transposed
    cache = (_Tensor((5, Hk, 64, D), torch.uint8), _Tensor((5, Hk, D, 64), torch.uint8), _Tensor((5, Hk, 2), torch.float32))
    out = _Tensor((Bn, Lq, Hq, D), torch.float16)
    table, lens = _Tensor((Bn, 1), torch.int32), _Tensor((Bn,), torch.int32)
    B.znni_kv8_attn(q, *cache, table, lens, 64, out=out, stream=side)
    assert log == [("copy", 77), ("launch", 77)]
    log.clear()
    B.znni_kv8_attn(q, *cache, table, lens, 64, out=out)
    assert log == [("copy", 0), ("launch", 0)]
    assert current == [0]


# ---- on the GPU: the current stream is busy while the call runs on another one ---------------------------------------

def _busy():
    torch.cuda._sleep(20_000_000)


def _ordered_side():
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    return side


def _cache_call(dtype=torch.bfloat16):
    Bn, Lq, Hq, Hk, D, n = 3, 2, 8, 2, 64, 300
    pools = B.kv8_alloc(20, Hk, D, DEV)
    k, v = (torch.randn(Bn * n, Hk, D, device=DEV).to(dtype) for _ in range(2))
    table = torch.arange(15, dtype=torch.int32, device=DEV).view(3, 5)
    cu = torch.arange(4, dtype=torch.int32, device=DEV) * n
    B.znni_kv8_append(*pools, k, v, table, cu, torch.zeros(3, dtype=torch.int32, device=DEV), n)
    q = torch.randn(Lq, Bn, Hq, D, device=DEV).to(dtype).transpose(0, 1)
    lens = torch.full((3,), n, dtype=torch.int32, device=DEV)
    return lambda **kw: B.znni_kv8_attn(q, *pools, table, lens, n, **kw)


def _window_call():
    q, k, v = (torch.randn(200, h, 64, device=DEV).bfloat16() for h in (8, 2, 2))
    cu = torch.tensor([0, 200], dtype=torch.int32, device=DEV)
    return lambda **kw: B.znni_attn_window(q, k, v, cu, cu, 200, 200, left=70, **kw)


def _rope_call():
    q = torch.randn(300, 8, 64, device=DEV).bfloat16()
    pos = torch.randint(0, 99, (300, 2), device=DEV, dtype=torch.int32)
    freq = torch.rand(32, device=DEV)
    return lambda **kw: B.znni_rope_axes(q, None, pos, freq, (16, 16), **kw)[0]


@pytest.mark.gpu
def test_uneven_queries_on_another_stream():
    call = _cache_call()
    want = call()
    for _ in range(3):
        side = _ordered_side()
        _busy()                                      # a copy on the current stream would come after the launch on `side`
        got = call(stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        del got


@pytest.mark.gpu
@pytest.mark.parametrize("make", [_cache_call, _window_call, _rope_call])
def test_results_on_another_stream_are_nobody_elses_memory(make):
    call = make()
    want = call()
    for _ in range(3):
        old = torch.empty_like(want)
        side = _ordered_side()
        _busy()
        old.fill_(float("nan"))                      # still to come when its memory is free again
        del old
        got = call(stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        # and the result's own memory is not given away while the current stream still reads it
        _busy()
        kept = got.clone()
        del got
        other = call(stream=side)
        with torch.cuda.stream(side):
            torch.empty_like(want).fill_(float("nan"))
        torch.cuda.synchronize()
        assert torch.equal(kept, want) and torch.equal(other, want)
        del kept, other
