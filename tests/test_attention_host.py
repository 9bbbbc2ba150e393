"""Refusals of the attention operators: every argument error is a status before any GPU work (addresses are made up and
never used), and the reference's own 8-bit rounding."""
import ctypes

import numpy as np
import pytest
import torch

import attention_ref as R
from paper_1606_05688_amd import binding as B

P, WS, BIG = 0x1000, 0x100000, 1 << 40
NULL, SHAPE, SIZE, WORKSPACE, FLAGS, ALIGN, TYPE = -1, -2, -3, -4, -5, -7, -8


def heads(data=P, token=256, head=64):
    return B._descriptor(data or 0, token, head)


def rope(type=B.BF16, T=4, Hq=2, Hk=1, D=64, q=True, k=True, pos=P, freq=P, axes=3, sections=(8, 8, 8), qo=True, ko=True, flags=0):
    h = {True: heads(), False: None}
    s = None if sections is None else (ctypes.c_int * 8)(*sections)
    return B.lib().znni_rope_axes(type, T, Hq, Hk, D, h.get(q, q), h.get(k, k), pos, freq, axes, s, h.get(qo, qo), h.get(ko, ko), flags, None)


@pytest.mark.parametrize("args,status", [
    (dict(q=False), NULL), (dict(k=False), NULL), (dict(qo=False), NULL), (dict(ko=False), NULL), (dict(sections=None), NULL),
    (dict(pos=None), NULL), (dict(freq=None), NULL), (dict(type=3), TYPE), (dict(type=-1), TYPE), (dict(flags=2), FLAGS),
    (dict(T=-1), SHAPE), (dict(Hq=0), SHAPE), (dict(Hk=-1), SHAPE), (dict(Hq=70000), SHAPE), (dict(D=0), SHAPE), (dict(axes=0), SHAPE),
    (dict(sections=(8, -1, 8)), SHAPE), (dict(sections=(16, 16, 1)), SHAPE), (dict(sections=(2147483647, 2147483647, 3)), SHAPE),
    (dict(D=60), SIZE), (dict(D=520), SIZE), (dict(axes=5), SIZE), (dict(pos=P + 2), ALIGN), (dict(freq=P + 1), ALIGN),
    (dict(T=0, pos=None), 0), (dict(T=0, q=True), 0),
])
def test_rope_refusals(args, status):
    assert rope(**args) == status


def test_heads_that_are_not_aligned():
    for bad in (heads(P + 8), heads(token=4), heads(head=12), heads(token=-4)):
        assert rope(q=bad) == ALIGN and rope(ko=bad) == ALIGN
        assert attn(k=bad) == ALIGN and attn(out=bad) == ALIGN
        assert append(v=bad) == ALIGN and kv8(q=bad) == ALIGN
    assert rope(q=heads(None)) == NULL and attn(v=heads(None)) == NULL and append(k=heads(None)) == NULL and kv8(out=heads(None)) == NULL


def attn(type=B.F16, Bn=2, Hq=4, Hk=2, D=64, q=True, k=True, v=True, cu_q=P, cu_k=P, mq=4000, mk=4000, left=9, right=0, sinks=0, out=True,
         ws=WS, wsb=BIG):
    h = {True: heads(), False: None}
    return B.lib().znni_attn_window(type, Bn, Hq, Hk, D, h.get(q, q), h.get(k, k), h.get(v, v), cu_q, cu_k, mq, mk, left, right, sinks, 1.0,
                                    h.get(out, out), ws, wsb, None)


COMMON = [
    (dict(type=9), TYPE), (dict(Hk=0), SHAPE), (dict(D=-8), SHAPE), (dict(Bn=-1), SHAPE), (dict(Bn=65536), SHAPE),
    (dict(D=4), SIZE), (dict(D=136), SIZE),
]


@pytest.mark.parametrize("args,status", COMMON + [
    (dict(q=False), NULL), (dict(k=False), NULL), (dict(v=False), NULL), (dict(out=False), NULL), (dict(cu_q=None), NULL), (dict(cu_k=None), NULL),
    (dict(Hq=5), SHAPE), (dict(mq=-1), SHAPE), (dict(mk=-1), SHAPE), (dict(left=-1), SHAPE), (dict(right=-1), SHAPE), (dict(sinks=-1), SHAPE),
    (dict(cu_k=P + 2), ALIGN), (dict(Bn=0, cu_q=None), 0), (dict(mq=0), 0),
])
def test_window_refusals(args, status):
    assert attn(**args) == status


def append(type=B.F16, Bn=2, Hk=2, D=64, k=True, v=True, cu=P, start=P, new=10, kc=P, vc=P, sc=P, pages=4, table=P, width=2):
    h = {True: heads(), False: None}
    return B.lib().znni_kv8_append(type, Bn, Hk, D, h.get(k, k), h.get(v, v), cu, start, new, kc, vc, sc, pages, table, width, None)


@pytest.mark.parametrize("args,status", COMMON + [
    (dict(k=False), NULL), (dict(v=False), NULL), (dict(cu=None), NULL), (dict(start=None), NULL), (dict(kc=None), NULL), (dict(vc=None), NULL),
    (dict(sc=None), NULL), (dict(table=None), NULL), (dict(new=-1), SHAPE), (dict(pages=-1), SHAPE), (dict(width=-1), SHAPE),
    (dict(kc=P + 8), ALIGN), (dict(vc=P + 4), ALIGN), (dict(sc=P + 4), ALIGN), (dict(table=P + 1), ALIGN), (dict(new=0, kc=None), 0),
    (dict(Bn=0), 0), (dict(width=0), 0), (dict(pages=0), 0),
])
def test_append_refusals(args, status):
    assert append(**args) == status


def kv8(type=B.F16, Bn=2, Lq=1, Hq=4, Hk=2, D=64, q=True, kc=P, vc=P, sc=P, pages=4, table=P, width=900, lens=P, mx=50000, left=B.ALL, sinks=0,
        out=True, ws=WS, wsb=BIG):
    h = {True: heads(), False: None}
    return B.lib().znni_kv8_attn(type, Bn, Lq, Hq, Hk, D, h.get(q, q), kc, vc, sc, pages, table, width, lens, mx, left, sinks, 1.0,
                                 h.get(out, out), ws, wsb, None)


@pytest.mark.parametrize("args,status", COMMON + [
    (dict(q=False), NULL), (dict(out=False), NULL), (dict(kc=None), NULL), (dict(vc=None), NULL), (dict(sc=None), NULL), (dict(table=None), NULL),
    (dict(lens=None), NULL), (dict(Hq=3), SHAPE), (dict(Lq=-1), SHAPE), (dict(mx=-1), SHAPE), (dict(left=-1), SHAPE), (dict(sinks=-2), SHAPE),
    (dict(pages=-1), SHAPE), (dict(width=-1), SHAPE), (dict(kc=P + 8), ALIGN), (dict(lens=P + 2), ALIGN), (dict(Lq=0), 0), (dict(Bn=0), 0),
])
def test_cache_attention_refusals(args, status):
    assert kv8(**args) == status


def test_workspaces():
    """Asked for twice they are the same, too little is refused, misaligned is refused; a null size pointer too."""
    b = ctypes.c_size_t(0)
    L = B.lib()
    assert L.znni_attn_window_workspace(B.F16, 1, 1, 1, 64, 1, 1, 1, 0, 0, None) == NULL
    assert L.znni_kv8_attn_workspace(B.F16, 1, 1, 1, 1, 64, 1, 1, 0, None) == NULL
    for mq, mk in ((1, 30000), (4000, 4000)):
        need = B.znni_attn_window_workspace(torch.float16, 2, 4, 2, 64, mq, mk, 2 ** 31 - 1, 0, 0)
        if need:
            assert attn(mq=mq, mk=mk, left=B.ALL, wsb=need - 1) == WORKSPACE and attn(mq=mq, mk=mk, left=B.ALL, ws=None) == NULL
            assert attn(mq=mq, mk=mk, left=B.ALL, ws=WS + 128) == ALIGN
    need = B.znni_kv8_attn_workspace(torch.float16, 2, 1, 4, 2, 64, 50000)
    if need:
        assert kv8(wsb=need - 1) == WORKSPACE and kv8(ws=None) == NULL and kv8(ws=WS + 128) == ALIGN
    with pytest.raises(B.ZnniError) as e:
        B.znni_kv8_attn_workspace(torch.float16, 2, 1, 4, 2, 200, 50000)
    assert e.value.status == SIZE


def test_workspace_of_the_largest_calls_does_not_overflow():
    """Sizes near the limits: a size that is right or a refusal, never a small number."""
    b = ctypes.c_size_t(0)
    for args in ((B.F32, 65535, 1, 65535, 1, 128, 2 ** 31 - 1, B.ALL, 0), (B.F32, 65535, 2 ** 31 - 1, 65535, 1, 128, 2 ** 31 - 1, B.ALL, 0)):
        assert B.lib().znni_kv8_attn_workspace(*args, ctypes.byref(b)) in (0, SHAPE)
        assert b.value < 1 << 62
    assert B.lib().znni_attn_window_workspace(B.F32, 65535, 65535, 1, 128, 2 ** 31 - 1, 2 ** 31 - 1, B.ALL, B.ALL, 0, ctypes.byref(b)) in (0, SHAPE)
    assert b.value < 1 << 62


def test_the_references_rounding_is_torchs():
    """e4m3 by the definition against torch's conversion on the CPU, ties and subnormals among the values."""
    r = np.random.default_rng(0)
    y = np.concatenate([r.standard_normal(20000) * 2.0 ** r.integers(-12, 8, 20000), (R._VALUES[1:] + R._VALUES[:-1]) / 2]).astype(np.float32)
    y = y[np.abs(y) <= 448]
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(R.to_e4m3(y), want.astype(np.float64))
    codes = torch.arange(256, dtype=torch.int64).to(torch.uint8)
    assert np.array_equal(R.e4m3(codes).numpy(), codes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
