"""The 8-bit cache: filling it against its definition (bit for bit), attention over it against the definition in 64 bits on
the values that the cache holds."""
import numpy as np
import pytest
import torch

import attention_ref as R
from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ALL = B.ALL
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _dev(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def _append(pools, ref, k, v, table, new, start):
    cu = np.concatenate([[0], np.cumsum(new)])
    B.znni_kv8_append(*pools, k.to(DEV), v.to(DEV), _dev(table), _dev(cu), _dev(start), max(new))
    ref.append(k.double().numpy(), v.double().numpy(), table, cu, start)


def _equal(pools, ref, table, lens):
    """All tokens of all sequences and the scales of their pages."""
    kc, vc, sc = (p.cpu() for p in pools)
    kv, vv = R.e4m3(kc).numpy(), R.e4m3(vc).numpy().transpose(0, 1, 3, 2)
    for b, n in enumerate(lens):
        for i in range(-(-int(n) // 64)):
            page, m = int(table[b, i]), min(64, int(n) - 64 * i)
            assert np.array_equal(sc[page].numpy().astype(np.float64), 2.0 ** ref.e[page].astype(np.float64)), (b, i)
            assert np.array_equal(kv[page][:, :m], ref.k[page][:, :m], equal_nan=True), (b, i, "keys")
            assert np.array_equal(vv[page][:, :m], ref.v[page][:, :m], equal_nan=True), (b, i, "values")


def _pools(pages, Hk, D, fill=255):
    return [p.view(torch.uint8).fill_(fill).view(p.dtype) for p in B.kv8_alloc(pages, Hk, D, DEV)]      # 255: codes and scales of NaN


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hk,D", [(1, 8), (3, 40), (2, 64), (4, 128), (2, 104)])
def test_appending_is_its_definition(dtype, Hk, D):
    print(f"[kv8] append {dtype} {Hk} {D}", flush=True)
    r = np.random.default_rng(D)
    Bn, width = 5, 6
    table = r.permutation(40)[:Bn * width].reshape(Bn, width)
    pools, ref = _pools(40, Hk, D), R.Cache(40, Hk, D)
    lens = np.zeros(Bn, dtype=np.int64)
    g = torch.Generator().manual_seed(D)
    # prompts, then single tokens, then a few, that grow and shrink by large factors: scales stay, or grow and move the old codes
    for step, new in enumerate([[0, 1, 63, 64, 130], [1, 1, 1, 1, 1], [1, 0, 2, 1, 3], [65, 64, 1, 100, 0], [1, 1, 1, 1, 1]]):
        size = (1.0, 0.01, 30.0, 1.0, 2000.0)[step]
        k, v = (size * torch.randn(sum(new), Hk, D, generator=g).to(dtype) for _ in range(2))
        k[:, :, ::3] *= 0.001                        # small values next to large ones: the type's subnormals
        _append(pools, ref, k, v, table, new, lens)
        lens += np.array(new)
        _equal(pools, ref, table, lens)
    used = table.ravel()
    rest = [p for p in range(40) if p not in used]
    assert all((p[rest].contiguous().view(torch.uint8) == 255).all() for p in pools)                     # other pages are not touched


def test_extreme_values_and_every_code():
    """Zeros, the largest and smallest values of fp32, infinities, NaN; every magnitude next to a tie."""
    Hk, D = 1, 128
    ties = (R._VALUES[1:] + R._VALUES[:-1]) / 2
    y = np.concatenate([R._VALUES, ties, np.nextafter(ties.astype(np.float32), np.float32(0)), np.nextafter(ties.astype(np.float32), np.float32(999))])
    y = np.concatenate([y, -y, [448.0] * 24]).astype(np.float32)
    pages = [np.zeros((64, 128)), np.resize(y, (64, 128)), np.resize(y * 2.0 ** -100, (64, 128)), np.resize(y * 2.0 ** 100, (64, 128)),
             np.full((64, 128), 3.4028235e38), np.full((64, 128), 1e-45), np.resize([np.inf, 1.0, -np.inf, np.nan, -2.5], (64, 128)),
             np.full((64, 128), np.nan), np.full((64, 128), -np.inf), np.resize([448.0, 448.00003], (64, 128))]
    x = torch.from_numpy(np.concatenate(pages).astype(np.float32))[:, None]
    n = len(pages)
    table = np.arange(n)[None]
    pools, ref = _pools(n, Hk, D), R.Cache(n, Hk, D)
    _append(pools, ref, x, -x, table, [64 * n], np.array([0]))
    _equal(pools, ref, table, [64 * n])


def test_bad_pages_are_dropped():
    """Entries outside the pools, tokens past the table: nothing is written for them, and attention does not see them."""
    Hk, D = 2, 32
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(300, Hk, D, generator=g) for _ in range(2))
    table = np.array([[2, -1, 9, 1]])
    pools, ref = _pools(4, Hk, D), R.Cache(4, Hk, D)
    _append(pools, ref, k, v, table, [300], np.array([0]))
    assert all((p[[0, 3]].contiguous().view(torch.uint8) == 255).all() for p in pools)
    q = torch.randn(1, 1, 2, D, generator=g)
    got = B.znni_kv8_attn(q.to(DEV), *pools, _dev(table), _dev([300]), 300)          # counts as 256: pages 0 and 3 of the table
    kk, vv = (torch.cat([ref.tokens(0, np.array([[p]]), 64, w) for p in (2, 1)]) for w in (0, 1))
    r = R.rows(q[0].double(), kk, vv, [127], ALL, 0, 0, D ** -0.5)
    R.check(got[0], r[0], R.bound(torch.float32, *r))


def _filled(seed, lens, Hk, D, dtype, spare=3):
    g = torch.Generator().manual_seed(seed)
    width = max(1, max(-(-n // 64) for n in lens)) + 1
    r = np.random.default_rng(seed)
    pages = len(lens) * width + spare
    table = r.permutation(pages)[:len(lens) * width].reshape(len(lens), width)
    pools, ref = _pools(pages, Hk, D), R.Cache(pages, Hk, D)
    k, v = (torch.randn(sum(lens), Hk, D, generator=g).to(dtype) for _ in range(2))
    _append(pools, ref, k, v, table, lens, np.zeros(len(lens), dtype=np.int64))
    return pools, ref, table


def _reference(q, ref, table, lens, left, sinks, scale):
    parts = []
    for b, n in enumerate(lens):
        pos = torch.arange(q.shape[1]) + n - q.shape[1]
        kk, vv = (ref.tokens(b, table, n, w) if n else torch.zeros(0, ref.k.shape[1], q.shape[3]).double() for w in (0, 1))
        parts.append(R.rows(q[b].double(), kk, vv, pos, left, 0, sinks, scale))
    return [torch.stack(p) for p in zip(*parts)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Hq,Hk,D,Lq,lens,left,sinks", [
    (1, 1, 8, 1, [1], ALL, 0),
    (4, 1, 64, 1, [63, 64, 65, 0, 1], ALL, 0),
    (16, 4, 128, 1, [777, 128], ALL, 0),
    (8, 2, 128, 1, [3000, 500, 64], 200, 4),
    (6, 2, 40, 3, [130, 2, 0, 65], 50, 0),              # fewer tokens than queries: rows before the first are zero
    (5, 5, 80, 2, [200, 129], 100, 70),
    (24, 1, 96, 2, [300], ALL, 0),                      # more rows than a tile of sixteen
    (3, 3, 24, 7, [500, 70], 63, 1),
    (40, 2, 32, 5, [90, 640], 10, 64),
    (2, 2, 112, 1, [1500], 0, 0),
    (7, 7, 16, 4, [260], 64, 128),
])
def test_attention_over_the_cache(dtype, Hq, Hk, D, Lq, lens, left, sinks):
    print(f"[kv8] attn {dtype} {(Hq, Hk, D, Lq, lens, left, sinks)}", flush=True)
    pools, ref, table = _filled(D + Lq, lens, Hk, D, dtype)
    q = torch.randn(len(lens), Lq, Hq, D, generator=torch.Generator().manual_seed(1)).to(dtype)
    r = _reference(q, ref, table, lens, left, sinks, D ** -0.5)
    args = (q.to(DEV), *pools, _dev(table), _dev(lens), max(lens))
    got = B.znni_kv8_attn(*args, left=left, sinks=sinks)
    R.check(got, r[0], R.bound(dtype, *r))
    assert torch.equal(got, B.znni_kv8_attn(*args, left=left, sinks=sinks))
    # a larger bound on the lengths may split the work otherwise, and moves results by rounding only
    R.check(B.znni_kv8_attn(*args[:-1], 100000, left=left, sinks=sinks), r[0], R.bound(dtype, *r))


def test_pages_that_no_row_sees_are_not_read():
    """Behind the window the table may name anything, and what a page holds past the last token is nobody's."""
    Hq, Hk, D, lens = 4, 2, 64, [1000]
    pools, ref, table = _filled(3, lens, Hk, D, torch.float32)
    q = torch.randn(1, 2, Hq, D, generator=torch.Generator().manual_seed(1))
    r = _reference(q, ref, table, lens, 150, 10, 0.125)
    cut = table.copy()
    cut[0, 1:13] = -7                                     # rows at 998 and 999 see 0 .. 9 and 848 .. : pages 0, 13, 14, 15
    cut[0, 16] = 1 << 30
    got = B.znni_kv8_attn(q.to(DEV), *pools, _dev(cut), _dev(lens), 1000, left=150, sinks=10, scale=0.125)
    R.check(got, r[0], R.bound(torch.float32, *r))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Lq", [1, 4])
def test_nan_codes_outside_a_rows_sight(dtype, Lq):
    """NaN among the window's pages but before the window, after a row's own position, and in sight of some rows only."""
    Hq, Hk, D, n, left = 4, 2, 64, 300, 100
    g = torch.Generator().manual_seed(2)
    k, v = (torch.randn(n, Hk, D, generator=g).to(dtype) for _ in range(2))
    k[194], v[195] = float("nan"), float("nan")           # the row at 299 sees 199 .. 299, that at 296 sees 196 ..
    v[197, 0, 3] = float("nan")                           # seen by rows 296 and 297 only
    k[298, 1, 9] = float("nan")                           # seen by rows 298 and 299, in one head
    v[299, 1, 60] = float("nan")
    table = np.arange(6)[None]
    pools, ref = _pools(6, Hk, D), R.Cache(6, Hk, D)
    _append(pools, ref, k, v, table, [n], np.array([0]))
    q = torch.randn(1, Lq, Hq, D, generator=g).to(dtype)
    r = _reference(q, ref, table, [n], left, 0, D ** -0.5)
    got = B.znni_kv8_attn(q.to(DEV), *pools, _dev(table), _dev([n]), n, left=left)
    fine = torch.isfinite(r[0])
    assert fine.any() and not fine.all()
    R.check(got, r[0], torch.where(fine, R.bound(dtype, *r), torch.ones_like(r[0])))


def test_long_cache_passes_32_bit_offsets():
    """A pool of more than 2^32 bytes whose last pages are the ones in use; sharp weights, many parts to join."""
    Hk, D, pages = 8, 128, 65536 + 200
    pools = B.kv8_alloc(pages, Hk, D, DEV)
    n = 100 * 64 - 5
    table = np.arange(pages - 100, pages)[None]
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(n, Hk, D, generator=g) for _ in range(2))
    k *= torch.linspace(0.1, 4, n)[:, None, None]
    B.znni_kv8_append(*pools, k.to(DEV), v.to(DEV), _dev(table), _dev([0, n]), _dev([0]), n)
    kc, vc, sc = (p[pages - 100:].cpu() for p in pools)
    kk = (R.e4m3(kc) * sc[:, :, 0, None, None].double()).permute(0, 2, 1, 3).reshape(-1, Hk, D)[:n]
    vv = (R.e4m3(vc) * sc[:, :, 1, None, None].double()).permute(0, 3, 1, 2).reshape(-1, Hk, D)[:n]
    assert (kk - k.double()).abs().max() <= 2.0 ** -4 * k.abs().max()
    q = torch.randn(1, 1, 32, D, generator=g)
    r = R.rows(q[0].double(), kk, vv, [n - 1], ALL, 0, 0, D ** -0.5)
    got = B.znni_kv8_attn(q.to(DEV), *pools, _dev(table), _dev([n]), n)
    R.check(got[0], r[0], R.bound(torch.float32, *r))


def test_streams_graphs_and_strided_queries():
    Hq, Hk, D, lens, dtype = 8, 2, 128, [700, 2500, 64], torch.bfloat16
    pools, ref, table = _filled(8, lens, Hk, D, dtype)
    t, l = _dev(table), _dev(lens)
    wide = torch.randn(3, 2, Hq + 4, D, device=DEV).to(dtype)
    q = wide[:, :, :Hq]
    want = B.znni_kv8_attn(q.contiguous(), *pools, t, l, 2500, left=900, sinks=2)
    assert torch.equal(B.znni_kv8_attn(q, *pools, t, l, 2500, left=900, sinks=2), want)
    assert torch.equal(B.znni_kv8_attn(q.transpose(0, 1).contiguous().transpose(0, 1), *pools, t, l, 2500, left=900, sinks=2), want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = B.znni_kv8_attn(q, *pools, t, l, 2500, left=900, sinks=2, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    # a step of serving in a graph: append a token, attend
    k, v = (torch.randn(3, Hk, D, device=DEV).to(dtype) for _ in range(2))
    cu, now = _dev([0, 1, 2, 3]), l - 1
    ws = torch.empty(max(256, B.znni_kv8_attn_workspace(dtype, 3, 2, Hq, Hk, D, 2500, 900, 2)), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.znni_kv8_append(*pools, k, v, t, cu, now, 1)
        B.znni_kv8_attn(q, *pools, t, l, 2500, left=900, sinks=2, out=out, workspace=ws)
    for turn in range(3):
        k.copy_(torch.randn(k.shape, device=DEV))
        wide.copy_(torch.randn(wide.shape, device=DEV))
        out.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        kept = [p.clone() for p in pools]
        B.znni_kv8_append(*pools, k, v, t, cu, now, 1)
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(kept, pools))
        assert torch.equal(out, B.znni_kv8_attn(q, *pools, t, l, 2500, left=900, sinks=2)), turn


def test_empty_calls():
    pools = _pools(2, 1, 16)
    none = torch.zeros(0, 1, 2, 16, device=DEV)
    t0 = torch.zeros(0, 3, dtype=torch.int32, device=DEV)
    assert B.znni_kv8_attn(none, *pools, t0, t0[:, 0].contiguous(), 0).shape == (0, 1, 2, 16)
    x = torch.ones(2, 1, 2, 16, device=DEV)
    assert (B.znni_kv8_attn(x, *pools, _dev([[0], [1]]), _dev([0, 0]), 0) == 0).all()
    assert (B.znni_kv8_attn(x, *pools, torch.zeros(2, 0, dtype=torch.int32, device=DEV), _dev([50, 1]), 50) == 0).all()
    k = torch.zeros(0, 1, 16, device=DEV)
    B.znni_kv8_append(*pools, k, k, _dev([[0], [1]]), _dev([0, 0, 0]), _dev([0, 5]), 0)
    B.znni_kv8_append(*pools, k, k, _dev([[0], [1]]), _dev([0, 0, 0]), _dev([0, 5]), 3)
    assert all((p.view(torch.uint8) == 255).all() for p in pools)
