"""Refusals of products with weights, norms between blocks and the gradients of windowed attention: every argument error is a status before any
GPU work (addresses are made up and never used), and arguments on another GPU are refused before the library is called."""
import ctypes

import pytest
import torch

from paper_1606_05688_amd import binding as B
from test_attention_devices import _Library, _On

P, WS, BIG = 0x1000, 0x100000, 1 << 50
NULL, SHAPE, SIZE, WORKSPACE, FLAGS, ALIGN, TYPE = -1, -2, -3, -4, -5, -7, -8


def rows(data=P, row=256):
    return B._rows_descriptor(data, row)


def heads(data=P, token=256, head=64):
    return B._descriptor(data, token, head)


def pick(x, default=None):
    return {True: rows() if default is None else default, False: None}.get(x, x)


def linear(type=B.BF16, M=8, N=16, K=64, x=True, w=True, bias=P, act=0, residual=True, z=True, out=True, ws=WS, wsb=BIG):
    return B.lib().znni_linear(type, M, N, K, pick(x), pick(w), bias, act, pick(residual), pick(z), pick(out), ws, wsb, None)


@pytest.mark.parametrize("args,status", [
    (dict(x=False), NULL), (dict(w=False), NULL), (dict(out=False), NULL), (dict(type=3), TYPE), (dict(act=-1), FLAGS), (dict(act=4), FLAGS),
    (dict(M=-1), SHAPE), (dict(N=-1), SHAPE), (dict(K=-1), SHAPE), (dict(N=1 << 27), SHAPE), (dict(K=1 << 27), SHAPE),
    (dict(x=rows(0)), NULL), (dict(w=rows(0)), NULL), (dict(out=rows(0)), NULL), (dict(residual=rows(0)), NULL), (dict(z=rows(0)), NULL),
    (dict(x=rows(P + 1)), ALIGN), (dict(out=rows(P + 1)), ALIGN), (dict(bias=P + 1), ALIGN), (dict(z=rows(P + 1)), ALIGN),
    (dict(type=B.F32, w=rows(P + 2)), ALIGN), (dict(out=rows(P, 15)), SHAPE), (dict(z=rows(P, 0)), SHAPE), (dict(out=rows(P, -16)), SHAPE),
    (dict(K=100000, ws=None), NULL), (dict(K=100000, wsb=16), WORKSPACE), (dict(K=100000, ws=WS + 8), ALIGN),
    (dict(M=0, x=rows(0), out=rows(0)), 0), (dict(N=0, w=rows(0), out=rows(0)), 0),
])
def test_linear_refusals(args, status):
    assert linear(**args) == status


def back(type=B.BF16, M=8, N=16, K=64, dout=True, x=True, w=True, z=True, act=2, dx=True, dw=True, dbias=P, ws=WS, wsb=BIG):
    return B.lib().znni_linear_backward(type, M, N, K, pick(dout), pick(x), pick(w), pick(z), act, pick(dx), pick(dw), dbias, ws, wsb, None)


@pytest.mark.parametrize("args,status", [
    (dict(dout=False), NULL), (dict(x=False), NULL), (dict(w=False), NULL), (dict(z=False), NULL), (dict(type=-1), TYPE), (dict(act=5), FLAGS),
    (dict(M=-2), SHAPE), (dict(dout=rows(0)), NULL), (dict(z=rows(0)), NULL), (dict(dx=rows(0)), NULL), (dict(dw=rows(0)), NULL),
    (dict(dout=rows(P + 1)), ALIGN), (dict(dbias=P + 1), ALIGN), (dict(dx=rows(P, 63)), SHAPE), (dict(dw=rows(P, 63)), SHAPE),
    (dict(ws=None), NULL), (dict(wsb=64), WORKSPACE), (dict(ws=WS + 128), ALIGN),
])
def test_linear_gradient_refusals(args, status):
    assert back(**args) == status


def test_linear_workspaces():
    b = ctypes.c_size_t(7)
    q = B.lib().znni_linear_backward_workspace
    assert q(B.BF16, 8, 16, 64, 2, 8, ctypes.byref(b)) == FLAGS and q(B.BF16, 8, 16, 64, 9, 1, ctypes.byref(b)) == FLAGS
    assert q(B.BF16, 8, 16, 64, 0, 1, None) == NULL and B.lib().znni_linear_workspace(B.BF16, 8, 16, 64, None) == NULL
    assert B.znni_linear_workspace(torch.bfloat16, 0, 16, 64) == 0
    # what goes into an activation is held for the products
    assert B.znni_linear_backward_workspace(torch.bfloat16, 1000, 77, 64, "gelu") >= 1000 * 80 * 2
    for M, N, K in ((1, 1, 1), (17, 4000, 90000), (1 << 20, 3, 64), (3, 1 << 20, 64)):
        for dtype in (torch.float32, torch.float16):
            for act in (None, "relu"):
                whole = B.znni_linear_backward_workspace(dtype, M, N, K, act)
                assert whole % 256 == 0 and all(B.znni_linear_backward_workspace(dtype, M, N, K, act, part) <= whole for part in (1, 2, 4))


def norm(type=B.BF16, T=8, C=64, x=True, y=True, gate=True, post=P, pre=P, flags=B.NORM_POST | B.NORM_PRE, h=True, z=True):
    return B.lib().znni_block_norm(type, T, C, pick(x), pick(y), pick(gate), post, pre, 1.0, 1e-5, flags, pick(h), pick(z), None)


@pytest.mark.parametrize("args,status", [
    (dict(x=False), NULL), (dict(h=False), NULL), (dict(z=False), NULL), (dict(y=False), NULL), (dict(type=9), TYPE), (dict(flags=16), FLAGS),
    (dict(T=-1), SHAPE), (dict(C=0), SHAPE), (dict(C=16385), SIZE), (dict(flags=B.NORM_POST), FLAGS), (dict(flags=B.NORM_PRE), FLAGS),
    (dict(gate=False, flags=B.NORM_POST | B.NORM_PRE | B.NORM_GATE_SHARED), FLAGS), (dict(y=False, h=False), FLAGS),
    (dict(y=False, h=False, gate=False, post=None, pre=None, z=False, flags=0), FLAGS), (dict(x=rows(0)), NULL), (dict(y=rows(0)), NULL),
    (dict(gate=rows(0)), NULL), (dict(z=rows(P + 1)), ALIGN), (dict(post=P + 1), ALIGN), (dict(pre=P + 1), ALIGN), (dict(h=rows(P, 63)), SHAPE),
    (dict(z=rows(P, -64)), SHAPE), (dict(T=0), 0),
])
def test_norm_refusals(args, status):
    assert norm(**args) == status


def norm_back(type=B.BF16, T=8, C=64, dh=True, dz=True, h=True, y=True, gate=True, post=P, pre=P, flags=B.NORM_POST | B.NORM_PRE, dx=True, dy=True,
              dgate=True, dpost=P, dpre=P, ws=WS, wsb=BIG):
    return B.lib().znni_block_norm_backward(type, T, C, pick(dh), pick(dz), pick(h), pick(y), pick(gate), post, pre, 1.0, 1e-5, flags, pick(dx),
                                            pick(dy), pick(dgate), dpost, dpre, ws, wsb, None)


@pytest.mark.parametrize("args,status", [
    (dict(dz=False), NULL), (dict(h=False), NULL), (dict(y=False), NULL), (dict(gate=False), NULL), (dict(type=3), TYPE), (dict(flags=32), FLAGS),
    (dict(C=-1), SHAPE), (dict(C=20000), SIZE), (dict(flags=B.NORM_POST), FLAGS), (dict(flags=B.NORM_PRE), FLAGS), (dict(dx=rows(P, 60)), SHAPE),
    (dict(dh=False, dz=False, pre=None, dpre=None, flags=B.NORM_POST), NULL), (dict(dgate=rows(0)), NULL), (dict(dy=rows(P + 1)), ALIGN),
    (dict(dpost=P + 1), ALIGN), (dict(ws=None), NULL), (dict(wsb=256), WORKSPACE), (dict(ws=WS + 4), ALIGN),
])
def test_norm_gradient_refusals(args, status):
    assert norm_back(**args) == status


def attn(type=B.F16, Bn=2, Hq=4, Hk=2, D=64, q=True, k=True, v=True, out=True, stats=P, dout=True, cu_q=P, cu_k=P, mq=4000, mk=4000, left=9, right=0,
         sinks=0, dq=True, dk=True, dv=True, ws=WS, wsb=BIG):
    h = [pick(x, heads()) for x in (q, k, v, out, dout, dq, dk, dv)]
    return B.lib().znni_attn_window_backward(type, Bn, Hq, Hk, D, h[0], h[1], h[2], h[3], stats, h[4], cu_q, cu_k, mq, mk, left, right, sinks, 1.0, h[5],
                                             h[6], h[7], ws, wsb, None)


@pytest.mark.parametrize("args,status", [
    (dict([(n, False)]), NULL) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")] + [
    (dict([(n, heads(0))]), NULL) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")] + [
    (dict([(n, heads(P + 8))]), ALIGN) for n in ("q", "k", "v", "out", "dout", "dq", "dk", "dv")] + [
    (dict([(n, heads(token=4))]), ALIGN) for n in ("q", "dout", "dk")] + [
    (dict(stats=None), NULL), (dict(stats=P + 4), ALIGN), (dict(cu_q=None), NULL), (dict(cu_k=P + 2), ALIGN), (dict(ws=None), NULL),
    (dict(wsb=100), WORKSPACE), (dict(ws=WS + 16), ALIGN), (dict(type=7), TYPE), (dict(Hk=3), SHAPE), (dict(D=12), SIZE), (dict(D=136), SIZE),
    (dict(Bn=70000), SHAPE), (dict(mq=-1), SHAPE), (dict(mk=-1), SHAPE), (dict(left=-1), SHAPE), (dict(right=-1), SHAPE), (dict(sinks=-1), SHAPE),
    (dict(mq=1 << 30, Hq=8), SHAPE), (dict(mk=B.ALL - 1), SHAPE), (dict(Bn=65535, mk=1 << 30), SHAPE),
    (dict(Bn=0), 0), (dict(mq=0, mk=0), 0),
])
def test_attention_gradient_refusals(args, status):
    assert attn(**args) == status


F, I, U, X = torch.float16, torch.int32, torch.uint8, torch.float32
CALLS = {
    "stats": (lambda a: B.znni_attn_window(a["q"], a["k"], a["v"], a["cu_q"], a["cu_k"], 6, 9, out=a["out"], workspace=a["ws"], stats=a["stats"]),
              dict(q=((6, 4, 32), F), k=((9, 2, 32), F), v=((9, 2, 32), F), cu_q=((2,), I), cu_k=((2,), I), out=((6, 4, 32), F), ws=((256,), U), stats=((6, 4, 2), X))),
    "attention": (lambda a: B.znni_attn_window_backward(a["dout"], a["q"], a["k"], a["v"], a["out"], a["stats"], a["cu_q"], a["cu_k"], 6, 9, dq=a["dq"],
                                                        dk=a["dk"], dv=a["dv"], workspace=a["ws"]),
                  dict(q=((6, 4, 32), F), k=((9, 2, 32), F), v=((9, 2, 32), F), out=((6, 4, 32), F), dout=((6, 4, 32), F), stats=((6, 4, 2), X), cu_q=((2,), I),
                       cu_k=((2,), I), dq=((6, 4, 32), F), dk=((9, 2, 32), F), dv=((9, 2, 32), F), ws=((1 << 20,), U))),
    "linear": (lambda a: B.znni_linear(a["x"], a["w"], a["b"], act="gelu", residual=a["r"], keep=a["z"], out=a["out"], workspace=a["ws"]),
               dict(x=((6, 32), F), w=((8, 32), F), b=((8,), F), r=((6, 8), F), z=((6, 8), F), out=((6, 8), F), ws=((256,), U))),
    "linear gradients": (lambda a: B.znni_linear_backward(a["dout"], a["x"], a["w"], z=a["z"], act="gelu", dx=a["dx"], dw=a["dw"], dbias=a["db"], workspace=a["ws"]),
                         dict(dout=((6, 8), F), x=((6, 32), F), w=((8, 32), F), z=((6, 8), F), dx=((6, 32), F), dw=((8, 32), F), db=((8,), F), ws=((1 << 20,), U))),
    "norm": (lambda a: B.znni_block_norm(a["x"], a["y"], gate=a["gate"], post=a["post"], pre=a["pre"], h=a["h"], z=a["z"]),
             dict(x=((6, 32), F), y=((6, 32), F), gate=((6, 32), F), post=((32,), F), pre=((32,), F), h=((6, 32), F), z=((6, 32), F))),
    "norm gradients": (lambda a: B.znni_block_norm_backward(a["dh"], a["dz"], a["h"], a["y"], gate=a["gate"], post=a["post"], pre=a["pre"], dx=a["dx"], dy=a["dy"],
                                                            dgate=a["dgate"], dpost=a["dpost"], dpre=a["dpre"], workspace=a["ws"]),
                       dict(h=((6, 32), F), dh=((6, 32), F), dz=((6, 32), F), y=((6, 32), F), gate=((32,), F), post=((32,), F), pre=((32,), F), dx=((6, 32), F),
                            dy=((6, 32), F), dgate=((32,), F), dpost=((32,), F), dpre=((32,), F), ws=((1 << 20,), U))),
}
FIRST = {"stats": "q", "attention": "q", "linear": "x", "linear gradients": "dout", "norm": "x", "norm gradients": "h"}


class _Shaped(_On):
    def dim(self):
        return len(self.shape)


def _call(monkeypatch, name, elsewhere=None, other=None):
    monkeypatch.setattr(B, "_lib", _Library())
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    _Library.called = False
    call, args = CALLS[name]
    call({n: _Shaped(1 if n == elsewhere else 0, a[0], other if n == elsewhere and other else a[1]) for n, a in args.items()})


@pytest.mark.parametrize("name", CALLS)
def test_all_on_one_gpu(monkeypatch, name):
    _call(monkeypatch, name)
    assert _Library.called


@pytest.mark.parametrize("name,argument", [(n, a) for n, (_, args) in CALLS.items() for a in args if a != FIRST[n]])
def test_one_on_another_gpu(monkeypatch, name, argument):
    with pytest.raises(AssertionError):
        _call(monkeypatch, name, argument)
    assert not _Library.called


@pytest.mark.parametrize("name,argument", [(n, a) for n, (_, args) in CALLS.items() for a in args if a != FIRST[n]])
def test_one_of_another_type(monkeypatch, name, argument):
    monkeypatch.setattr(_Shaped, "__init__", lambda self, gpu, shape, dtype: _On.__init__(self, 0, shape, dtype))
    with pytest.raises(AssertionError):
        _call(monkeypatch, name, argument, torch.float64)
    assert not _Library.called
