"""Gradients of windowed attention against the definition in 64 bits: types, head widths and groups, windows, first tokens, ragged and empty
sequences, rows that see nothing, walks that are split, strides, what is not finite, scales, graphs."""
import pytest
import torch

import attention_back_ref as R
from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ALL = B.ALL


def starts(lens):
    return [sum(lens[:i]) for i in range(len(lens) + 1)]


def make(lens, Hq, Hk, D, dtype, seed=0, behind=0, by=1.0):
    g = torch.Generator().manual_seed(seed)
    cq, ck = starts([a for a, _ in lens]), starts([b for _, b in lens])
    r = lambda n, H: (torch.randn((n + behind, H, D), generator=g, dtype=torch.float64) * by).to(dtype).cuda()  # noqa: E731
    q, k, v, dout = r(cq[-1], Hq), r(ck[-1], Hk), r(ck[-1], Hk), r(cq[-1], Hq)
    i = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return (q, k, v, dout), (i(cq), i(ck), max(a for a, _ in lens), max(b for _, b in lens))


def call(tensors, where, left, right, sinks, scale=None, **kw):
    q, k, v, dout = tensors
    out, stats = B.znni_attn_window(q, k, v, *where, left=left, right=right, sinks=sinks, scale=scale, stats=True)
    return out, stats, B.znni_attn_window_backward(dout, q, k, v, out, stats, *where, left=left, right=right, sinks=sinks, scale=scale, **kw)


def compare(lens, tensors, left, right, sinks, got, scale=None, what=""):
    q, k, v, dout = (x.double().cpu() for x in tensors)
    cq, ck = starts([a for a, _ in lens]), starts([b for _, b in lens])
    for s in range(len(lens)):
        a, b = slice(cq[s], cq[s + 1]), slice(ck[s], ck[s + 1])
        exp = R.backward(q[a], k[b], v[b], dout[a], left, right, sinks, q.shape[2] ** -0.5 if scale is None else scale, tensors[0].dtype)
        for name, y, rows, e in zip(("dq", "dk", "dv"), got, (a, b, b), exp):
            R.check(y[rows], *e, f"{what} sequence {s} {name}")


CASES = [
    ([(1, 1)], 1, 1, 8, ALL, 0, 0),
    ([(5, 5)], 2, 1, 64, ALL, 0, 0),
    ([(40, 40), (1, 33), (0, 7), (7, 0), (0, 0), (64, 65)], 4, 2, 64, ALL, 0, 0),
    ([(130, 130)], 4, 4, 128, 30, 0, 0),
    ([(200, 200)], 8, 2, 128, 50, 0, 3),
    ([(150, 170), (33, 400)], 6, 2, 40, 20, 10, 4),
    ([(90, 60), (70, 3)], 3, 3, 24, ALL, 0, 0),                 # the first rows see nothing
    ([(90, 60)], 5, 1, 96, 10, ALL, 0),
    ([(100, 100)], 3, 1, 72, ALL, ALL, 0),
    ([(257, 257)], 1, 1, 32, 0, 0, 0),                           # each sees itself
    ([(10, 1000)], 4, 2, 56, 20, 0, 4),                          # first tokens far before the window
    ([(700, 700)], 2, 1, 64, 20, 0, 5),                          # rows past the window of first tokens: workgroups of their own
    ([(600, 600), (300, 300)], 2, 2, 16, 5, 3, 200),             # more first tokens than a tile has keys
    ([(4, 2500)], 4, 1, 128, ALL, 0, 0),                         # the walk over the keys is split
    ([(2000, 40)], 4, 1, 80, ALL, ALL, 0),                       # the walk over the rows is split
    ([(1200, 130)], 2, 1, 128, 7, ALL, 3),
    ([(33, 64)], 128, 1, 32, ALL, 0, 0),                         # more heads to a key head than a tile has rows
    ([(20, 30)], 48, 3, 88, 12, 2, 1),
    ([(1, 77)] * 9, 16, 4, 128, ALL, 0, 0),
    ([(200, 200)], 2, 2, 104, ALL, ALL, 0),
    ([(200, 200)], 2, 1, 112, ALL, 0, 0),
    ([(200, 200)], 2, 2, 120, 90, 0, 0),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_cases(dtype, case):
    lens, Hq, Hk, D, left, right, sinks = CASES[case]
    tensors, where = make(lens, Hq, Hk, D, dtype, case)
    out, stats, got = call(tensors, where, left, right, sinks)
    assert torch.equal(out, B.znni_attn_window(*tensors[:3], *where, left=left, right=right, sinks=sinks))
    compare(lens, tensors, left, right, sinks, got)
    q, k, v, _ = (x.double().cpu() for x in tensors)
    cq, ck = starts([a for a, _ in lens]), starts([b for _, b in lens])
    for s in range(len(lens)):
        exp = R.forward(q[cq[s]:cq[s + 1]], k[ck[s]:ck[s + 1]], v[ck[s]:ck[s + 1]], left, right, sinks, D ** -0.5)[0]
        # weights rounded to the type, sums of up to 2500 terms of size 4 in fp32, the result rounded
        assert (out[cq[s]:cq[s + 1]].double().cpu() - exp).abs().sum() <= 4 * exp.numel() * (2 * R.UNIT[dtype] + 2500 * 2.0 ** -23)


@pytest.mark.parametrize("dtype", TYPES)
def test_statistics(dtype):
    for case in (2, 5, 6, 13):
        lens, Hq, Hk, D, left, right, sinks = CASES[case]
        tensors, where = make(lens, Hq, Hk, D, dtype, 50 + case)
        _, stats, _ = call(tensors, where, left, right, sinks)
        q, k, v, _ = (x.double().cpu() for x in tensors)
        cq, ck = starts([a for a, _ in lens]), starts([b for _, b in lens])
        for s in range(len(lens)):
            a, b = slice(cq[s], cq[s + 1]), slice(ck[s], ck[s + 1])
            _, total, top = R.forward(q[a], k[b], v[b], left, right, sinks, D ** -0.5)
            ref, got = stats[a, :, 0].double().cpu() * D ** -0.5, stats[a, :, 1].double().cpu()
            assert torch.equal(got == 0, total == 0) and torch.isfinite(ref).all()
            there = total > 0
            off = (torch.log(got) + ref - torch.log(total) - top).abs()[there]
            # a score is off by (D + 8) 2^-24 of sum |q||k|, at most about 30 here; the sum by 1 + count of 2^-23
            assert off.numel() == 0 or off.max() < (D + 8) * 2.0 ** -24 * 30 + 3000 * 2.0 ** -23


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(dtype, scale):
    lens, left, right, sinks = [(70, 90), (33, 20)], 25, 4, 2
    tensors, where = make(lens, 4, 2, 48, dtype, 3)
    _, _, got = call(tensors, where, left, right, sinks, scale)
    compare(lens, tensors, left, right, sinks, got, scale, f"scale {scale}")


@pytest.mark.parametrize("dtype", TYPES)
def test_large_scores(dtype):
    """Scores of some thousands: their differences are what counts.  Inputs are whole numbers, so that scores are exact."""
    lens, left, right, sinks = [(100, 120)], 60, 0, 1
    tensors, where = make(lens, 2, 1, 32, dtype, 4)
    q, k, v, dout = tensors
    q.copy_((q * 4).round()), k.copy_((k * 4).round())
    q[..., 0], k[..., 0] = 60, 60
    _, _, got = call(tensors, where, left, right, sinks, 1.0)
    compare(lens, tensors, left, right, sinks, got, 1.0)


@pytest.mark.parametrize("by", [2.0 ** -14, 2.0 ** -7, 2.0 ** 6, 2.0 ** 9])
def test_sizes_of_gradients_in_fp16(by):
    """Gradients of a result that are small or large: what is rounded on the way keeps the type's bits."""
    lens, left, right, sinks = [(300, 1500)], ALL, 0, 0
    tensors, where = make(lens, 2, 1, 64, torch.float16, 5)
    tensors[3].mul_(by)
    _, _, got = call(tensors, where, left, right, sinks)
    compare(lens, tensors, left, right, sinks, got, what=f"{by}")


@pytest.mark.parametrize("dtype", TYPES)
def test_strides(dtype):
    lens, Hq, Hk, D = [(70, 70), (40, 90)], 4, 2, 40
    (q, k, v, dout), where = make(lens, Hq, Hk, D, dtype, 6)
    out, stats, got = call((q, k, v, dout), where, 30, 2, 3)
    wide = lambda x: torch.full((x.shape[0], x.shape[1] + 1, D + 8), float("nan"), dtype=dtype, device="cuda")[:, 1:, 8:].copy_(x)  # noqa: E731
    turned = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    for form in (wide, turned):
        a, b, c, e, o = (form(x) for x in (q, k, v, dout, out))
        outs = [form(torch.zeros_like(x)) for x in (q, k, v)]
        again = B.znni_attn_window_backward(e, a, b, c, o, stats, *where, left=30, right=2, sinks=3, dq=outs[0], dk=outs[1], dv=outs[2])
        assert all(torch.equal(x, y) and x is z for x, y, z in zip(again, got, outs))
    assert torch.isnan(wide(q)._base[:, 0]).all()
    # one set of values for all tokens, and its own head for all heads
    same_v, same_d = v[:1].expand(v.shape), dout[:, :1].expand(dout.shape)
    out, stats, got = call((q, k, same_v, same_d), where, 30, 2, 3)
    compare(lens, (q, k, same_v, same_d), 30, 2, 3, got)


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_behind_the_last_sequence_stays(dtype):
    lens = [(30, 50), (17, 9)]
    tensors, where = make(lens, 4, 2, 64, dtype, 7, behind=11)
    outs = [torch.full_like(x, 7) for x in tensors[:3]]
    _, _, got = call(tensors, where, 20, 0, 0, dq=outs[0], dk=outs[1], dv=outs[2])
    compare(lens, tensors, 20, 0, 0, got)
    for y, n in zip(got, (47, 59, 59)):
        assert (y[n:] == 7).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("case", [4, 5, 9, 11, 15])
def test_not_finite(dtype, bad, case):
    """What is not finite in a row or key has no influence on keys that the row does not see and rows that do not see the key."""
    lens, Hq, Hk, D, left, right, sinks = CASES[case]
    tensors, where = make(lens, Hq, Hk, D, dtype, 20 + case)
    nq, nk = lens[0]
    q, k, v, dout = (x.double().cpu()[:n] for x, n in zip(tensors, (nq, nk, nk, nq)))
    plain = R.backward(q, k, v, dout, left, right, sinks, D ** -0.5, dtype)
    see = R.seen(nq, nk, left, right, sinks)
    for which, token, d in ((0, nq // 2, 3), (1, nk // 2, 5), (2, nk // 2 + 1, D - 1), (3, nq // 2 + 1, 0), (1, nk - 1, 0), (3, 0, 1)):
        mine = [x.clone() for x in tensors]
        mine[which][token, 0, d] = bad
        _, _, got = call(mine, where, left, right, sinks)
        rows = see[:, token] if which in (1, 2) else torch.arange(nq) == token          # that it may touch
        keys = see[rows].any(0)
        # head 0 of the queries, and of the keys; other query heads of key head 0 if it is a key's or value's
        heads = Hq // Hk if which in (1, 2) else 1
        free_q = torch.ones(nq, Hq, dtype=torch.bool)
        free_q[rows.nonzero()[:, 0], :heads] = False
        free_k = torch.ones(nk, Hk, dtype=torch.bool)
        free_k[keys.nonzero()[:, 0], 0] = False
        for y, (e, bound), free in zip(got, plain, (free_q, free_k, free_k)):
            R.check(y.cpu()[:len(free)][free], e[free], bound[free], f"{which} {token}")
        # and what the formula makes of it is not finite
        if bad != bad and rows.any() and keys.any():
            if which in (0, 1):
                assert torch.isnan(got[1][:nk][keys.cuda(), 0]).all() and torch.isnan(got[2][:nk][keys.cuda(), 0]).all()
            if which == 3:
                assert torch.isnan(got[0][token, 0]).all() and torch.isnan(got[2][:nk][keys.cuda(), 0, d]).all()
                others = [e for e in range(D) if e != d]
                R.check(got[2][:nk][:, 0, others], plain[2][0][:, 0, others], plain[2][1][:, 0, others])


@pytest.mark.parametrize("dtype", TYPES)
def test_graph_and_streams(dtype):
    """A captured call, replayed between eager ones of the same tensors; two graphs with one workspace, one after the other."""
    lens, left, right, sinks = [(130, 300), (64, 64), (1, 500)], 70, 0, 6
    tensors, where = make(lens, 4, 2, 64, dtype, 8)
    q, k, v, dout = tensors
    kw = dict(left=left, right=right, sinks=sinks)
    ws = torch.empty(max(B.znni_attn_window_workspace(dtype, 3, 4, 2, 64, *where[2:], **kw), B.znni_attn_window_backward_workspace(dtype, 3, 4, 2, 64, *where[2:], **kw)),
                     dtype=torch.uint8, device="cuda")
    bufs = [torch.empty_like(x) for x in (q, q, k, v)] + [torch.empty((q.shape[0], 4, 2), device="cuda")]

    def step(out, dq, dk, dv, stats, **more):
        B.znni_attn_window(q, k, v, *where, out=out, stats=stats, workspace=ws, **kw, **more)
        B.znni_attn_window_backward(dout, q, k, v, out, stats, *where, dq=dq, dk=dk, dv=dv, workspace=ws, **kw, **more)

    step(*bufs)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            step(*bufs)
    for i in range(3):
        for x in tensors:
            x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(i)))
        eager = [torch.empty_like(x) for x in bufs]
        step(*eager)
        torch.cuda.synchronize()
        for graph in graphs:
            for x in bufs:
                x.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, bufs))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    out, stats = B.znni_attn_window(q, k, v, *where, stats=True, stream=st, **kw)
    got = B.znni_attn_window_backward(dout, q, k, v, out, stats, *where, stream=st, **kw)
    torch.cuda.current_stream().wait_stream(st)
    assert all(torch.equal(a, b) for a, b in zip(eager, (out, *got, stats)))


def test_against_differences():
    lens = [(9, 12), (6, 4)]
    (q, k, v, dout), where = make(lens, 4, 2, 16, torch.float32, 9)
    kw = dict(left=5, right=1, sinks=1)
    _, _, grads = call((q, k, v, dout), where, 5, 1, 1)
    g = torch.Generator().manual_seed(1)
    for n, grad in enumerate(grads):
        way, f = torch.randn(grad.shape, generator=g).cuda(), []
        for s in (-1, 1):
            t = [x + s * 2.0 ** -7 * way if i == n else x for i, x in enumerate((q, k, v))]
            f.append((B.znni_attn_window(*t, *where, **kw).double() * dout.double()).sum())
        off = abs((f[1] - f[0]).item() * 2.0 ** 6 - (grad.double() * way.double()).sum().item())
        # third derivatives: at most some ten times (scale |q| |way|)^3 of a row of values up to 4; sums of 960 results, each off by 2^-21
        assert off <= dout.abs().sum().item() * 4 * (10 * 4.0 ** 3 * 2.0 ** -14 / 6 + 2.0 ** -21 * 2.0 ** 6)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_far_apart(dtype):
    """Strides past what 32-bit offsets hold within a tile, tokens past 2^31 elements."""
    lens = [(600, 600)]
    (q, k, v, dout), where = make(lens, 2, 2, 32, dtype, 12)
    out, stats, got = call((q, k, v, dout), where, 100, 0, 2)

    def apart(x):
        y = torch.empty_strided(x.shape, ((1 << 22) + 64, 32, 1), dtype=dtype, device="cuda")
        return y.copy_(x)

    for i in range(3):                               # keys and values, queries and the result's gradient, what is written
        a = [apart(x) if (i == 0 and n in (1, 2)) or (i == 1 and n in (0, 3)) else x for n, x in enumerate((q, k, v, dout))]
        kw = dict(dq=apart(q), dk=apart(k), dv=apart(v)) if i == 2 else {}
        again = B.znni_attn_window_backward(a[3], *a[:3], out, stats, *where, left=100, sinks=2, **kw)
        assert all(torch.equal(x, y) for x, y in zip(again, got))
        del a, kw, again
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_and_heads_backwards(dtype):
    """Strides below zero, in what is read."""
    lens, Hq, Hk, D = [(70, 70), (40, 90)], 4, 2, 40
    (q, k, v, dout), (cu_q, cu_k, mq, mk) = make(lens, Hq, Hk, D, dtype, 13)
    out, stats, got = call((q, k, v, dout), (cu_q, cu_k, mq, mk), 30, 2, 3)
    size = q.element_size()
    held = []

    def backwards(x):
        y = x.flip(0, 1).contiguous()
        held.append(y)
        T, H, _ = x.shape
        return B._descriptor(y.data_ptr() + (T * H - 1) * D * size, -H * D, -D)

    new = [torch.empty_like(x) for x in (q, k, v)]
    there = [B._descriptor(x.data_ptr(), x.shape[1] * D, D) for x in new]
    ws = torch.empty(B.znni_attn_window_backward_workspace(dtype, 2, Hq, Hk, D, mq, mk, 30, 2, 3), dtype=torch.uint8, device="cuda")
    status = B.lib().znni_attn_window_backward(B._TYPES[dtype], 2, Hq, Hk, D, backwards(q), backwards(k), backwards(v), backwards(out), stats.data_ptr(),
                                               backwards(dout), cu_q.data_ptr(), cu_k.data_ptr(), mq, mk, 30, 2, 3, D ** -0.5, *there, ws.data_ptr(),
                                               ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert status == 0
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(new, got))


@pytest.mark.parametrize("dtype", TYPES)
def test_fewer_rows_and_keys_than_the_call_says(dtype):
    """max_q and max_k are bounds: larger ones change the launch, not the result's meaning; rows past a smaller max_q take no part."""
    lens = [(50, 80), (3, 3)]
    tensors, (cu_q, cu_k, mq, mk) = make(lens, 4, 2, 64, dtype, 14)
    out, stats, _ = call(tensors, (cu_q, cu_k, mq, mk), 20, 0, 2)
    q, k, v, dout = tensors
    got = B.znni_attn_window_backward(dout, q, k, v, out, stats, cu_q, cu_k, 5000, 9000, left=20, sinks=2)
    compare(lens, tensors, 20, 0, 2, got)


def test_a_call_of_keys_without_rows():
    for dtype in TYPES:
        (q, k, v, dout), where = make([(0, 70), (0, 0), (0, 5)], 2, 1, 64, dtype, 15)
        out, stats, got = call((q, k, v, dout), where, 5, 0, 3)
        assert got[0].shape == (0, 2, 64) and (got[1] == 0).all() and (got[2] == 0).all()
