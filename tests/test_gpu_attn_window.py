"""Attention with a sliding window and first tokens that stay visible, against the definition in 64 bits."""
import pytest
import torch

import attention_ref as R
from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ALL = B.ALL
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _starts(n):
    return [sum(n[:i]) for i in range(len(n) + 1)]


def _reference(q, k, v, nq, nk, left, right, sinks, scale):
    parts = []
    cq, ck = _starts(nq), _starts(nk)
    for b in range(len(nq)):
        pos = torch.arange(nq[b]) + nk[b] - nq[b]
        parts.append(R.rows(q[cq[b]:cq[b + 1]].double(), k[ck[b]:ck[b + 1]].double(), v[ck[b]:ck[b + 1]].double(), pos, left, right, sinks, scale))
    return [torch.cat(p) for p in zip(*parts)]


def _run(q, k, v, nq, nk, left, right, sinks, scale=None, **kw):
    cu = [torch.tensor(_starts(n), dtype=torch.int32, device=DEV) for n in (nq, nk)]
    return B.znni_attn_window(q, k, v, cu[0], cu[1], max(nq), max(nk), left=left, right=right, sinks=sinks, scale=scale, **kw)


def _inputs(seed, nq, nk, Hq, Hk, D, dtype):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(sum(nq), Hq, D, generator=g).to(dtype), torch.randn(sum(nk), Hk, D, generator=g).to(dtype),
            torch.randn(sum(nk), Hk, D, generator=g).to(dtype))


CASES = [
    # (Hq, Hk, D, queries, keys, left, right, sinks)
    (1, 1, 8, [1], [1], ALL, 0, 0),
    (2, 1, 64, [65], [65], ALL, 0, 0),
    (4, 2, 128, [130, 1, 0, 64], [130, 200, 5, 64], 40, 0, 4),
    (8, 8, 64, [63, 64, 65, 3], [63, 64, 65, 0], 16, 0, 1),
    (3, 1, 40, [100, 7], [300, 129], 70, 30, 5),
    (5, 5, 80, [33], [257], 0, 0, 0),
    (6, 2, 96, [90], [90], 20, ALL, 100),
    (4, 4, 32, [128], [128], ALL, ALL, 0),
    (16, 1, 128, [5, 9], [700, 64], 300, 0, 16),
    (2, 2, 24, [200], [60], 30, 0, 2),                 # more queries than keys: the first see nothing
    (7, 7, 120, [50, 50], [50, 51], 0, 3, 70),
    (10, 2, 16, [1, 1, 1], [1, 64, 1000], ALL, 0, 0),
    (12, 4, 104, [2, 4], [513, 66], 500, 2, 3),
    (40, 1, 64, [11], [150], 64, 0, 64),               # window and sinks that touch
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c[:3]) + f"-{len(c[3])}x{c[3][0]}")
def test_against_the_definition(dtype, case):
    Hq, Hk, D, nq, nk, left, right, sinks = case
    print(f"[attn] {dtype} {case}", flush=True)
    q, k, v = _inputs(sum(nq) + D, nq, nk, Hq, Hk, D, dtype)
    ref = _reference(q, k, v, nq, nk, left, right, sinks, D ** -0.5)
    got = _run(q.to(DEV), k.to(DEV), v.to(DEV), nq, nk, left, right, sinks)
    R.check(got, ref[0], R.bound(dtype, *ref), str(case))
    again = _run(q.to(DEV), k.to(DEV), v.to(DEV), nq, nk, left, right, sinks)
    assert torch.equal(got, again)


def _many(x, n, copies):
    """The sequences of n tokens, one behind the other, so many times over."""
    return x.repeat(copies, 1, 1), n * copies


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", [c for c in CASES if sum(c[3]) < 400], ids=lambda c: "-".join(str(x) for x in c[:3]) + f"-{len(c[3])}x{c[3][0]}")
def test_many_sequences(dtype, case):
    """So many row tiles that no keys are shared out: every copy of a sequence has the definition's result, and the same one."""
    Hq, Hk, D, nq, nk, left, right, sinks = case
    copies = 400 // (Hk * len(nq)) + 1
    print(f"[attn many] {dtype} {case} {copies}", flush=True)
    q, k, v = _inputs(sum(nq) + D + 1, nq, nk, Hq, Hk, D, dtype)
    ref = _reference(q, k, v, nq, nk, left, right, sinks, D ** -0.5)
    (qs, nqs), (ks, nks), (vs, _) = _many(q, nq, copies), _many(k, nk, copies), _many(v, nk, copies)
    got = _run(qs.to(DEV), ks.to(DEV), vs.to(DEV), nqs, nks, left, right, sinks).view(copies, sum(nq), Hq, D)
    assert torch.equal(got, got[:1].expand_as(got))
    R.check(got[0], ref[0], R.bound(dtype, *ref), str(case))


@pytest.mark.parametrize("D", [8, 32, 40, 72, 96, 104, 128])
@pytest.mark.parametrize("nq,Hq", [(1, 1), (1, 8), (7, 4), (33, 1), (129, 3), (450, 5)])
def test_few_rows_in_fp32(nq, Hq, D):
    """Workgroups whose waves share the elements of a head, and (450 rows of five heads) those whose waves do not."""
    nk, left, sinks = [nq + 301], 150, 5
    print(f"[attn few] {nq} {Hq} {D}", flush=True)
    q, k, v = _inputs(nq + D, [nq], nk, Hq, 1, D, torch.float32)
    v[nq // 2, 0, D - 1] = float("inf")             # seen by some rows of long ones, by none of a single one
    ref = _reference(q, k, v, [nq], nk, left, 2, sinks, D ** -0.5)
    clean = torch.isfinite(ref[0])
    got = _run(q.to(DEV), k.to(DEV), v.to(DEV), [nq], nk, left, 2, sinks)
    R.check(got, ref[0], torch.where(clean, R.bound(torch.float32, *ref), torch.ones_like(ref[0])))


def test_more_workgroups_than_a_dimension_of_a_launch_holds():
    """Many sequences under a bound on their length that is far too large: most workgroups have nothing to do."""
    n, D = 65535, 8
    q, k, v = (x.to(DEV) for x in _inputs(5, [n], [n], 1, 1, D, torch.bfloat16))
    cu = torch.arange(n + 1, dtype=torch.int32, device=DEV)
    few = B.znni_attn_window(q, k, v, cu, cu, 1, 1)
    assert torch.equal(few, v)                      # a row's only key is its own
    assert torch.equal(B.znni_attn_window(q, k, v, cu, cu, 128 * 130, 1), few)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("copies", [1, 210])
def test_values_that_are_not_finite_in_both_halves_of_a_tile(dtype, copies):
    """Infinities that some rows of a tile see and others do not, few rows (two waves share them) and many."""
    Hq, Hk, D, n, left = 2, 2, 64, 90, 20
    q, k, v = _inputs(12, [n], [n], Hq, Hk, D, dtype)
    for j, e in ((3, 0), (40, 9), (50, 33), (70, 63), (89, 5)):
        v[j, j % 2, e] = float("inf") if j % 4 else float("-inf")
    ref = _reference(q, k, v, [n], [n], left, 0, 2, D ** -0.5)
    (qs, nq), (ks, nk), (vs, _) = _many(q, [n], copies), _many(k, [n], copies), _many(v, [n], copies)
    got = _run(qs.to(DEV), ks.to(DEV), vs.to(DEV), nq, nk, left, 0, 2).view(copies, n, Hq, D)
    assert torch.equal(got, got[:1].expand_as(got))
    clean = torch.isfinite(ref[0])
    assert clean.any() and not clean.all() and not torch.isnan(ref[0]).any()
    R.check(got[0], ref[0], torch.where(clean, R.bound(dtype, *ref), torch.ones_like(ref[0])))


@pytest.mark.parametrize("dtype", TYPES)
def test_long_sequences_and_sharp_weights(dtype):
    """Many tiles, scores far apart: the running maximum moves late in the sequence, most weights vanish."""
    Hq, Hk, D, nq, nk = 2, 1, 64, [40], [5000]
    q, k, v = _inputs(3, nq, nk, Hq, Hk, D, dtype)
    k = (k.float() * torch.linspace(0.1, 6, 5000)[:, None, None]).to(dtype)
    for left, sinks in ((ALL, 0), (3000, 8), (100, 200)):
        ref = _reference(q, k, v, nq, nk, left, 0, sinks, 0.4)
        R.check(_run(q.to(DEV), k.to(DEV), v.to(DEV), nq, nk, left, 0, sinks, scale=0.4), ref[0], R.bound(dtype, *ref), f"{left} {sinks}")
    one = _run(q[:1].to(DEV), k.to(DEV), v.to(DEV), [1], nk, ALL, 0, 0, scale=0.4)
    ref = _reference(q[:1], k, v, [1], nk, ALL, 0, 0, 0.4)
    R.check(one, ref[0], R.bound(dtype, *ref), "one row")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D", [8, 40, 64, 72, 128])
@pytest.mark.parametrize("n", [600, 1100, 2500])
def test_keys_shared_by_workgroups(dtype, D, n):
    """Two to twenty parts a row, of heads of all widths; one sequence is so short that most of its parts are empty."""
    Hq, Hk, nq, nk = 6, 2, [33, 1, 2], [n, n - 100, 2]
    print(f"[attn parts] {dtype} {D} {n}", flush=True)
    q, k, v = _inputs(n + D, nq, nk, Hq, Hk, D, dtype)
    for left, sinks in ((ALL, 0), (n // 2, 70)):
        ref = _reference(q, k, v, nq, nk, left, 0, sinks, D ** -0.5)
        R.check(_run(q.to(DEV), k.to(DEV), v.to(DEV), nq, nk, left, 0, sinks), ref[0], R.bound(dtype, *ref), f"{left} {sinks}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("nq", [1, 70])
def test_what_a_row_does_not_see_has_no_influence(dtype, nq):
    """NaN and infinities in keys and values behind a row's window, before it and beside the sequence; rows that see one take it."""
    Hq, Hk, D, nk = 4, 2, 64, 400
    q, k, v = _inputs(9, [nq], [nk], Hq, Hk, D, dtype)
    pad_k, pad_v = torch.full((nk + 40, Hk, D), float("nan")).to(dtype), torch.full((nk + 40, Hk, D), float("inf")).to(dtype)
    left, sinks = 60, 3
    k[100:200] = float("nan")                       # rows 330.. - 60 never get there
    v[150:250] = float("inf")
    v[330 + 35, 1, 5] = float("inf")                # seen by some rows of the 70, by the one only if its window holds it
    v[330 - 50, 0, 7] = float("nan")
    k[330 + 20, 0, 3] = float("nan")
    pad_k[20:20 + nk], pad_v[20:20 + nk] = k, v
    # the definition, touching only what is seen: NaN and infinities as arithmetic has them
    ref = _reference(q, k, v, [nq], [nk], left, 0, sinks, D ** -0.5)
    cu_k = torch.tensor([20, 20 + nk], dtype=torch.int32, device=DEV)
    cu_q = torch.tensor([0, nq], dtype=torch.int32, device=DEV)
    got = B.znni_attn_window(q.to(DEV), pad_k.to(DEV), pad_v.to(DEV), cu_q, cu_k, nq, nk, left=left, sinks=sinks)
    clean = torch.isfinite(ref[0])
    assert clean.any() and (nq == 1 or not clean.all())
    tol = torch.where(clean, R.bound(dtype, *ref), torch.ones_like(ref[0]))
    R.check(got, ref[0], tol)


def test_scores_of_minus_infinity_and_of_the_lowest_value():
    """Keys of the type's lowest value: weights that vanish, and rows all of whose weights do."""
    D = 16
    q = torch.zeros(3, 1, D)
    q[:, 0, 0] = torch.tensor([1.0, 2.0, 3.0])
    k, v = torch.zeros(3, 1, D), torch.randn(3, 1, D, generator=torch.Generator().manual_seed(1))
    k[0, 0, 0] = float("-inf")
    k[1, 0, 0] = torch.finfo(torch.float32).min
    got = _run(q.to(DEV), k.to(DEV), v.to(DEV), [3], [3], ALL, 0, 0, scale=1.0).cpu()
    assert torch.equal(got[0], torch.zeros(1, D))           # its only key has no weight
    assert torch.isfinite(got[2]).all() and torch.equal(got[2], v[2])
    low = torch.full((4, 1, D), torch.finfo(torch.bfloat16).min).bfloat16()
    x = torch.zeros(4, 1, D).bfloat16()
    x[:, 0, 0] = 1
    got = _run(x.to(DEV), low.to(DEV), v[:1].expand(4, 1, D).bfloat16().to(DEV), [4], [4], ALL, 0, 0, scale=1e-3).cpu()
    assert torch.equal(got, v[:1].expand(4, 1, D).bfloat16())           # equal weights however low the scores


def test_strides_and_shared_heads():
    g = torch.Generator().manual_seed(4)
    T, H, D, dtype = 150, 4, 64, torch.bfloat16
    packed = torch.randn(T, 3 * H, D, generator=g).to(dtype)
    q, k, v = packed[:, :H], packed[:, H:2 * H], packed[:, 2 * H:]
    ref = _reference(q, k, v, [T], [T], 50, 0, 2, D ** -0.5)
    dev = packed.to(DEV)
    out = torch.full((H, T, D), float("nan"), dtype=dtype, device=DEV)
    _run(dev[:, :H], dev[:, H:2 * H], dev[:, 2 * H:], [T], [T], 50, 0, 2, out=out.transpose(0, 1))
    R.check(out.transpose(0, 1), ref[0], R.bound(dtype, *ref))
    # heads of keys and values that are one head, by a stride of zero
    one = dev[:, H:H + 1].expand(T, H, D)
    shared = _run(dev[:, :H], one, one, [T], [T], 50, 0, 2)
    ref = _reference(q, k[:, :1], k[:, :1], [T], [T], 50, 0, 2, D ** -0.5)
    R.check(shared, ref[0], R.bound(dtype, *ref))
    # keys in reverse order, by a negative stride, which torch does not have: sequences in the other order instead
    back = torch.flip(dev[:, H:2 * H], (0,)).flip((0,))
    assert torch.equal(_run(dev[:, :H], back, dev[:, 2 * H:], [T], [T], 50, 0, 2), out.transpose(0, 1))


def test_rows_beyond_the_stated_maximum_stay_and_empty_calls():
    q, k, v = (x.to(DEV) for x in _inputs(1, [30], [30], 2, 2, 32, torch.float16))
    cu = torch.tensor([0, 30], dtype=torch.int32, device=DEV)
    out = torch.full_like(q, 7.0)
    B.znni_attn_window(q, k, v, cu, cu, 10, 30, out=out)
    full = B.znni_attn_window(q, k, v, cu, cu, 30, 30)
    assert torch.equal(out[:10], full[:10]) and (out[10:] == 7).all()
    empty = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert B.znni_attn_window(q[:0], k[:0], v[:0], empty, empty, 0, 0).shape == (0, 2, 32)
    none = torch.tensor([0, 0], dtype=torch.int32, device=DEV)
    assert (B.znni_attn_window(q, k[:0], v[:0], cu, none, 30, 0) == 0).all()


@pytest.mark.parametrize("nq,nk", [([1, 1], [900, 3000]), ([200], [200])])
def test_other_streams_and_graphs(nq, nk):
    Hq, Hk, D, dtype = 8, 2, 128, torch.bfloat16
    q, k, v = (x.to(DEV) for x in _inputs(6, nq, nk, Hq, Hk, D, dtype))
    want = _run(q, k, v, nq, nk, 700, 0, 4)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = _run(q, k, v, nq, nk, 700, 0, 4, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    cu = [torch.tensor(_starts(n), dtype=torch.int32, device=DEV) for n in (nq, nk)]
    out = torch.empty_like(want)
    need = B.znni_attn_window_workspace(dtype, len(nq), Hq, Hk, D, max(nq), max(nk), 700, 0, 4)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.znni_attn_window(q, k, v, cu[0], cu[1], max(nq), max(nk), left=700, sinks=4, out=out, workspace=ws)
    for turn in range(3):
        q.copy_(torch.randn(q.shape, device=DEV))
        out.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, _run(q, k, v, nq, nk, 700, 0, 4)), turn
