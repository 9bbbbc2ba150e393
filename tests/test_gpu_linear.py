"""Products with weights against the definition in 64 bits: types, activations, sizes that end inside tiles, vectors and chunks, strides,
addresses that are not aligned, split sums, gradients, graphs."""
import pytest
import torch

import block_ref as R
from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def matrix(g, rows, cols, dtype, pad=0, shift=0, by=1.0):
    """A [rows, cols] tensor whose rows lie `pad` elements further apart, `shift` elements into its memory; NaN around it."""
    memory = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=dtype)
    x = memory.as_strided((rows, cols), (cols + pad, 1), shift)
    x.copy_(torch.randn((rows, cols), generator=g, dtype=torch.float64) * by)
    return memory.cuda().as_strided((rows, cols), (cols + pad, 1), shift)


def inputs(M, N, K, dtype, seed=0, pad=0, shift=0):
    g = torch.Generator().manual_seed(seed)
    return (matrix(g, M, K, dtype, pad, shift), matrix(g, N, K, dtype, pad, shift, max(K, 1) ** -0.5), (torch.randn(N, generator=g) * 0.3).to(dtype).cuda(),
            matrix(g, M, N, dtype, pad, shift), matrix(g, M, N, dtype, pad, shift))


def d(x):
    return None if x is None else x.double().cpu()


SIZES = [(1, 1, 1), (1, 64, 64), (3, 5, 7), (8, 136, 72), (16, 257, 513), (17, 33, 65), (64, 64, 64), (65, 129, 191), (130, 72, 1000), (200, 200, 200),
         (1, 300, 2500), (31, 8, 4097), (257, 40, 24), (128, 512, 96), (0, 5, 7), (5, 0, 7), (5, 7, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_sizes(dtype, M, N, K):
    x, w, bias, residual, _ = inputs(M, N, K, dtype)
    for kind, b, r in ((None, None, None), ("gelu", bias, residual), ("relu", bias, None), ("silu", None, residual)):
        out, z = B.znni_linear(x, w, b, act=kind, residual=r, keep=True)
        o, bo, zz, bz = R.linear(d(x), d(w), d(b), kind, d(r), dtype)
        R.check(out, o, bo, f"{kind}")
        R.check(z, zz, bz, f"{kind} z")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gradients(dtype, M, N, K):
    x, w, _, z, dout = inputs(M, N, K, dtype, 1)
    for kind in (None, "gelu", "relu", "silu"):
        got = B.znni_linear_backward(dout, x, w, z=None if kind is None else z, act=kind)
        for name, y, (e, b) in zip(("dx", "dw", "dbias"), got, R.linear_back(d(dout), d(x), d(w), d(z), kind, dtype)):
            R.check(y, e, b, f"{kind} {name}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (8, 8), (8, 1)])
def test_rows_apart_and_not_aligned(dtype, pad, shift):
    M, N, K = 70, 136, 200
    x, w, bias, residual, dout = inputs(M, N, K, dtype, 2, pad, shift)
    out = matrix(torch.Generator().manual_seed(9), M, N, dtype, pad, shift)
    assert B.znni_linear(x, w, bias, act="gelu", residual=residual, out=out) is out
    o, bo, _, _ = R.linear(d(x), d(w), d(bias), "gelu", d(residual), dtype)
    R.check(out, o, bo)
    dx, dw = matrix(torch.Generator().manual_seed(9), M, K, dtype, pad, shift), matrix(torch.Generator().manual_seed(9), N, K, dtype, pad, shift)
    got = B.znni_linear_backward(dout, x, w, z=residual, act="silu", dx=dx, dw=dw)
    for y, (e, b) in zip(got, R.linear_back(d(dout), d(x), d(w), d(residual), "silu", dtype)):
        R.check(y, e, b)
    for y in (out, dx, dw):          # what lies between the rows stays as it was
        if pad:
            rows, cols = y.shape
            assert torch.isnan(y.as_strided((rows, pad), (cols + pad, 1), shift + cols)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_one_row_read_many_times(dtype):
    x, w, _, _, dout = inputs(40, 48, 64, dtype, 3)
    same = x[5:6].expand(40, 64)
    o, bo, _, _ = R.linear(d(same), d(w), None, None, None, dtype)
    R.check(B.znni_linear(same, w), o, bo)
    back = x.flip(0)
    got = B.znni_linear_backward(dout[3:4].expand(40, 48), back, w)
    for y, (e, b) in zip(got, R.linear_back(d(dout[3:4].expand(40, 48)), d(back), d(w), None, None, dtype)):
        R.check(y, e, b)


def test_residual_in_place_and_parts_of_the_gradients():
    x, w, bias, residual, dout = inputs(100, 72, 80, torch.bfloat16, 4)
    expected = B.znni_linear(x, w, bias, act="silu", residual=residual)
    mine = residual.clone()
    assert torch.equal(B.znni_linear(x, w, bias, act="silu", residual=mine, out=mine), expected)
    whole = B.znni_linear_backward(dout, x, w, z=residual, act="gelu")
    for want in ((True, False, False), (False, True, False), (False, False, True)):
        got = B.znni_linear_backward(dout, x, w, z=residual, act="gelu", inputs=want[0], weights=want[1], bias=want[2])
        for y, e, has in zip(got, whole, want):
            assert torch.equal(y, e) if has else y is None


@pytest.mark.parametrize("dtype", TYPES)
def test_larger_tiles(dtype):
    """Enough rows and columns for every tile size; some of the rows and columns are checked."""
    for M, N, K in ((2304, 1160, 136), (4100, 4360, 72)):
        x, w, bias, residual, _ = inputs(M, N, K, dtype, 5)
        out = B.znni_linear(x, w, bias, act="relu", residual=residual)
        rows, cols = torch.arange(0, M, 37), torch.arange(0, N, 31)
        o, bo, _, _ = R.linear(d(x)[rows], d(w), d(bias), "relu", d(residual)[rows], dtype)
        R.check(out[rows.cuda()], o, bo)
        dx, dw, _ = B.znni_linear_backward(residual, x, w, bias=False)
        (e, b), _, _ = R.linear_back(d(residual)[rows], d(x)[rows], d(w), None, None, dtype)
        R.check(dx[rows.cuda()], e, b)
        _, (e, b), _ = R.linear_back(d(residual)[:, cols], d(x), d(w)[cols], None, None, dtype)
        R.check(dw[cols.cuda()], e, b)


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan_go_where_the_formula_takes_them(dtype):
    x, w, _, _, dout = inputs(70, 80, 72, dtype, 6)
    plain = B.znni_linear(x, w)
    grads = B.znni_linear_backward(dout, x, w)
    x[3, 5], x[40, 70] = float("inf"), float("nan")
    dout[7, 9] = float("nan")
    out = B.znni_linear(x, w)
    rest = [m for m in range(70) if m not in (3, 40)]
    assert torch.equal(out[rest], plain[rest]) and torch.isnan(out[40]).all()
    assert torch.equal(out[3] > 0, w[:, 5] > 0) and torch.isinf(out[3]).all()
    dx, dw, db = B.znni_linear_backward(dout, x, w)
    rest = [m for m in range(70) if m != 7]
    assert torch.equal(dx[rest], grads[0][rest]) and torch.isnan(dx[7]).all()
    assert torch.isnan(dw[9]).all() and torch.isnan(db[9]) and torch.isnan(db).sum() == 1
    rest, cols = [n for n in range(80) if n != 9], [k for k in range(72) if k not in (5, 70)]
    assert torch.equal(dw[rest][:, cols], grads[1][rest][:, cols]) and not torch.isfinite(dw[:, [5, 70]]).any()


@pytest.mark.parametrize("M,N,K", [(4, 520, 1000), (300, 64, 4000), (600, 700, 128)])
def test_graph(M, N, K):
    """Captured, replayed with new inputs between eager calls; workspaces of the caller."""
    dtype = torch.bfloat16
    x, w, bias, z, dout = inputs(M, N, K, dtype, 7)
    ws = torch.empty(max(B.znni_linear_workspace(dtype, M, N, K), B.znni_linear_backward_workspace(dtype, M, N, K, "gelu"), 256), dtype=torch.uint8, device="cuda")
    out, kept = torch.empty_like(z), torch.empty_like(z)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(bias)

    def step(o, k, a, b, c):
        B.znni_linear(x, w, bias, act="gelu", keep=k, out=o, workspace=ws)
        B.znni_linear_backward(dout, x, w, z=k, act="gelu", dx=a, dw=b, dbias=c, workspace=ws)

    step(out, kept, dx, dw, db)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, kept, dx, dw, db)
    for i in range(3):
        x.copy_(torch.randn(M, K, generator=torch.Generator().manual_seed(i)))
        eager = [torch.empty_like(y) for y in (out, kept, dx, dw, db)]
        step(*eager)
        torch.cuda.synchronize()
        for y in (out, kept, dx, dw, db):
            y.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (out, kept, dx, dw, db)))


def test_another_stream():
    x, w, bias, z, dout = inputs(200, 130, 96, torch.float16, 8)
    a = [B.znni_linear(x, w, bias, act="gelu"), *B.znni_linear_backward(dout, x, w, z=z, act="gelu")]
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    b = [B.znni_linear(x, w, bias, act="gelu", stream=st), *B.znni_linear_backward(dout, x, w, z=z, act="gelu", stream=st)]
    torch.cuda.current_stream().wait_stream(st)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_gradients_against_differences():
    g = torch.Generator().manual_seed(11)
    x, w, bias = (torch.randn(s, generator=g).cuda() for s in ((6, 10), (9, 10), (9,)))
    dout = torch.randn((6, 9), generator=g).cuda()
    for kind in ("gelu", "silu"):
        _, z = B.znni_linear(x, w, bias, act=kind, keep=True)
        grads = B.znni_linear_backward(dout, x, w, z=z, act=kind)
        for t, dt in zip((x, w, bias), grads):
            way = torch.randn(t.shape, generator=g).cuda()
            f = []
            for s in (-1, 1):
                moved = [t + s * 2.0 ** -6 * way if y is t else y for y in (x, w, bias)]
                f.append((B.znni_linear(*moved, act=kind).double() * dout.double()).sum())
            # second differences: a third derivative of order 1 times step^2, sums of 54 fp32 results over the step
            size = (dout.abs().sum() * way.abs().sum()).item()
            assert abs((f[1] - f[0]).item() * 2.0 ** 5 - (dt.double() * way.double()).sum().item()) <= size * (2.0 ** -12 + 2.0 ** -24 * 20 * 2.0 ** 6)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_far_apart(dtype):
    """Row strides past what 32-bit offsets hold within a tile, elements past 2^31."""
    M, N, K = 600, 72, 40
    x, w, bias, residual, dout = inputs(M, N, K, dtype, 12)
    far = torch.empty_strided((M, K), (1 << 22, 1), dtype=dtype, device="cuda").copy_(x)
    assert torch.equal(B.znni_linear(far, w, bias), B.znni_linear(x, w, bias))
    a, b = B.znni_linear_backward(dout, far, w), B.znni_linear_backward(dout, x, w)
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    far.fill_(7)
    assert torch.equal(B.znni_linear_backward(dout, x, w, dx=far)[0], b[0])


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_backwards(dtype):
    """Row strides below zero, in what is read."""
    M, N, K = 70, 40, 64
    x, w, bias, _, dout = inputs(M, N, K, dtype, 13)
    y = x.flip(0).contiguous()
    out, dw = torch.empty_like(dout), torch.empty_like(w)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    back = B._rows_descriptor(y.data_ptr() + (M - 1) * K * y.element_size(), -K)
    r = lambda t: B._rows_descriptor(t.data_ptr(), t.shape[1])  # noqa: E731
    st = torch.cuda.current_stream().cuda_stream
    assert B.lib().znni_linear(B._TYPES[dtype], M, N, K, back, r(w), bias.data_ptr(), 0, None, None, r(out), ws.data_ptr(), ws.numel(), st) == 0
    assert B.lib().znni_linear_backward(B._TYPES[dtype], M, N, K, r(dout), back, None, None, 0, None, r(dw), None, ws.data_ptr(), ws.numel(), st) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, B.znni_linear(x, w, bias)) and torch.equal(dw, B.znni_linear_backward(dout, x, w)[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_activations_over_their_range(dtype):
    """Values from the smallest to the largest, through a product with ones."""
    z = torch.cat([s * torch.logspace(-30, 30 if dtype != torch.float16 else 4, 401, base=10, dtype=torch.float64) for s in (1, -1)]
                  + [torch.linspace(-16, 16, 2001, dtype=torch.float64)]).to(dtype).cuda()[:, None]
    one = torch.ones((1, 1), dtype=dtype, device="cuda")
    for kind in ("relu", "gelu", "silu"):
        o, bo, _, _ = R.linear(d(z), d(one), None, kind, None, dtype)
        R.check(B.znni_linear(z, one, act=kind), o, bo, kind)
        dx, _, _ = B.znni_linear_backward(torch.ones_like(z), z, one, z=z, act=kind, weights=False, bias=False)
        _, s = R.act(d(z), kind)
        # a slope is made of functions off by 8 half steps of fp32, times |z| where it is not yet constant (|z| up to 100)
        tol = R.UNIT[dtype] * s.abs() + 8 * R.E * (d(z).abs().clamp(max=100) + 1) + R.TINY[dtype]
        R.check(dx, s, tol * (1 + R.UNIT[dtype]), kind + " slope")
