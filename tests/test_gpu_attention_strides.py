"""Heads of tokens in any order and far apart: strides that are negative, zero, or too large for 32-bit offsets, against the same
call on the same values side by side."""
import struct

import pytest
import torch

from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _heads(x, token=1, head=1):
    """The znni_heads of x [T, H, D], contiguous, with its tokens or heads (-1) from the last to the first."""
    T, H, D = x.shape
    at = (T - 1) * H * D * (token < 0) + (H - 1) * D * (head < 0)
    return B._descriptor(x.data_ptr() + at * x.element_size(), token * H * D, head * D)


def _turned(x, token, head):
    return x.flip([d for d, s in ((0, token), (1, head)) if s < 0]).contiguous()


def _stream():
    return torch.cuda.current_stream().cuda_stream


SIGNS = [(-1, 1), (1, -1), (-1, -1)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("signs", SIGNS)
@pytest.mark.parametrize("T,Hq,Hk,D,R", [(300, 4, 2, 64, 24), (1, 3, 1, 40, 20), (2000, 6, 6, 128, 64)])
def test_positions_of_heads_from_the_last_to_the_first(dtype, signs, T, Hq, Hk, D, R):
    q, k = (torch.randn(T, h, D, device=DEV).to(dtype) for h in (Hq, Hk))
    pos = torch.randint(-99, 99, (T, 1), device=DEV, dtype=torch.int32)
    freq = torch.rand(R, device=DEV)
    want = B.znni_rope_axes(_turned(q, *signs), _turned(k, *signs), pos, freq, (R,))
    got = [torch.full_like(x, float("nan")) for x in (q, k)]
    status = B.lib().znni_rope_axes(B._TYPES[dtype], T, Hq, Hk, D, _heads(q, *signs), _heads(k, *signs), pos.data_ptr(), freq.data_ptr(), 1,
                                    struct.pack("i", R), _heads(got[0]), _heads(got[1]), 0, _stream())
    assert status == 0 and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("signs", SIGNS)
@pytest.mark.parametrize("nq,nk,Hq,Hk,D", [([1], [900], 4, 2, 128), ([200, 7], [200, 130], 6, 3, 64), ([3000], [3000], 8, 4, 32), ([40], [333], 2, 1, 40),
                                           ([5000], [5000], 4, 2, 128)])
def test_window_over_heads_from_the_last_to_the_first(dtype, signs, nq, nk, Hq, Hk, D):
    q, k, v = (torch.randn(sum(n), h, D, device=DEV).to(dtype) for n, h in ((nq, Hq), (nk, Hk), (nk, Hk)))
    cu = [torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device=DEV) for n in (nq, nk)]
    want = B.znni_attn_window(*(_turned(x, *signs) for x in (q, k, v)), *cu, max(nq), max(nk), left=150, sinks=3, scale=0.125)
    out = torch.full_like(q, float("nan"))
    need = B.znni_attn_window_workspace(dtype, len(nq), Hq, Hk, D, max(nq), max(nk), 150, 0, 3)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    status = B.lib().znni_attn_window(B._TYPES[dtype], len(nq), Hq, Hk, D, *(_heads(x, *signs) for x in (q, k, v)), cu[0].data_ptr(), cu[1].data_ptr(),
                                      max(nq), max(nk), 150, 0, 3, 0.125, _heads(out), ws.data_ptr(), ws.numel(), _stream())
    assert status == 0 and torch.equal(out, want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("signs", SIGNS)
def test_cache_from_heads_from_the_last_to_the_first(dtype, signs):
    """Appending, then attention of queries in that order."""
    n, Hq, Hk, D, Lq = 300, 4, 2, 64, 3
    k, v = (torch.randn(n, Hk, D, device=DEV).to(dtype) for _ in range(2))
    q = torch.randn(Lq, Hq, D, device=DEV).to(dtype)
    table = torch.arange(5, dtype=torch.int32, device=DEV)[None]
    cu, start = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, n], [0]))
    one, two = ([p.view(torch.uint8).fill_(0).view(p.dtype) for p in B.kv8_alloc(5, Hk, D, DEV)] for _ in range(2))
    B.znni_kv8_append(*one, _turned(k, *signs), _turned(v, *signs), table, cu, start, n)
    status = B.lib().znni_kv8_append(B._TYPES[dtype], 1, Hk, D, _heads(k, *signs), _heads(v, *signs), cu.data_ptr(), start.data_ptr(), n,
                                     *(p.data_ptr() for p in two), 5, table.data_ptr(), 5, _stream())
    assert status == 0 and all(torch.equal(a, b) for a, b in zip(one, two))
    want = B.znni_kv8_attn(_turned(q, *signs)[None], *one, table, cu[1:], n, left=200)[0]
    out = torch.full_like(q, float("nan"))
    need = B.znni_kv8_attn_workspace(dtype, 1, Lq, Hq, Hk, D, n, 200)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    status = B.lib().znni_kv8_attn(B._TYPES[dtype], 1, Lq, Hq, Hk, D, _heads(q, *signs), *(p.data_ptr() for p in one), 5, table.data_ptr(), 5,
                                   cu[1:].data_ptr(), n, 200, 0, D ** -0.5, _heads(out), ws.data_ptr(), ws.numel(), _stream())
    assert status == 0 and torch.equal(out, want)


def _apart(x, memory, at, token):
    """x [T, H, D] in `memory`, tokens that many elements apart."""
    T, H, D = x.shape
    y = memory.as_strided((T, H, D), (token, D, 1), at)
    return y.copy_(x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("token", [(1 << 22) - 8, 1 << 22, (1 << 22) + 8, (1 << 26) + 8])
def test_tokens_far_apart(dtype, token):
    """Offsets within a tile that fit 32 bits and that do not, tokens whose offset passes 2^32 bytes."""
    T, Hq, Hk, D = 150 if token < 1 << 25 else 70, 4, 2, 64
    memory = torch.empty(T * token + 4096, dtype=dtype, device=DEV)
    q, k, v = (torch.randn(T, h, D, device=DEV).to(dtype) for h in (Hq, Hk, Hk))
    cu = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    pos = torch.randint(-99, 99, (T, 1), device=DEV, dtype=torch.int32)
    freq = torch.rand(32, device=DEV)
    far = [_apart(x, memory, at, token) for x, at in ((q, 0), (k, 512), (v, 1024))]
    assert torch.equal(B.znni_attn_window(*far, cu, cu, T, T, left=90), B.znni_attn_window(q, k, v, cu, cu, T, T, left=90))
    assert all(torch.equal(a, b) for a, b in zip(B.znni_rope_axes(far[0], far[1], pos, freq, (32,)), B.znni_rope_axes(q, k, pos, freq, (32,))))
    out = memory.as_strided((T, Hq, D), (token, D, 1), 2048)
    B.znni_attn_window(q, k, v, cu, cu, T, T, left=90, out=out)
    assert torch.equal(out, B.znni_attn_window(q, k, v, cu, cu, T, T, left=90))
    table = torch.arange(3, dtype=torch.int32, device=DEV)[None]
    start = torch.zeros(1, dtype=torch.int32, device=DEV)
    one, two = ([p.view(torch.uint8).fill_(0).view(p.dtype) for p in B.kv8_alloc(3, Hk, D, DEV)] for _ in range(2))
    B.znni_kv8_append(*one, k, v, table, cu, start, T)
    B.znni_kv8_append(*two, far[1], far[2], table, cu, start, T)
    assert all(torch.equal(a, b) for a, b in zip(one, two))
    few = q[:7].view(7, 1, Hq, D)
    rows = far[0][:7].view(7, 1, Hq, D)
    t7, l7 = table.expand(7, 3).contiguous(), cu[1:].expand(7).contiguous()
    assert torch.equal(B.znni_kv8_attn(rows, *one, t7, l7, T), B.znni_kv8_attn(few, *one, t7, l7, T))


@pytest.mark.parametrize("dtype", TYPES)
def test_one_token_for_all(dtype):
    """A stride of zero: every token is the same one."""
    T, Hq, Hk, D = 200, 4, 2, 64
    k, v = (torch.randn(1, Hk, D, device=DEV).to(dtype).expand(T, Hk, D) for _ in range(2))
    q = torch.randn(1, Hq, D, device=DEV).to(dtype).expand(T, Hq, D)
    cu = torch.tensor([0, T], dtype=torch.int32, device=DEV)
    got = B.znni_attn_window(q, k, v, cu, cu, T, T, left=60)
    assert torch.equal(got, B.znni_attn_window(q.contiguous(), k.contiguous(), v.contiguous(), cu, cu, T, T, left=60))
    pos = torch.arange(T, device=DEV, dtype=torch.int32)[:, None]
    freq = torch.rand(20, device=DEV)
    assert torch.equal(B.znni_rope_axes(q, None, pos, freq, (20,))[0], B.znni_rope_axes(q.contiguous(), None, pos, freq, (20,))[0])
