"""Products on the larger tiles, 128 x 128 and 256 x 256, in all three forms (forward, dx, dw), every element against the definition in 64 bits: whole and
ragged rows, columns and steps, padded rows, addresses that are not aligned.  Which tiles a case takes is checked without a GPU (test_block_launches_host.py)."""
import pytest
import torch

import block_ref as R
from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]

# M, N, K, padding of rows, first element, and the tiles (64, 128, 256) of forward, dx and dw in 16-bit types and in fp32
CASES = [
    (2304, 2304, 2304, 0, 0, (128, 128, 128), (128, 128, 128)),
    (2296, 2312, 2328, 8, 8, (128, 128, 128), (128, 128, 128)),          # whole chunks of 16 bytes, tiles and steps that end early
    (2301, 2310, 2295, 0, 0, (128, 128, 128), (128, 128, 128)),          # by way of registers
    (2305, 2303, 2201, 3, 1, (128, 128, 128), (128, 128, 128)),
    (4096, 4096, 4096, 0, 0, (256, 256, 256), (128, 128, 128)),
    (4088, 4072, 4080, 16, 8, (256, 256, 256), (128, 128, 128)),
    (4093, 4090, 4085, 0, 0, (256, 256, 256), (128, 128, 128)),
    (4001, 4095, 4083, 5, 3, (256, 256, 256), (128, 128, 128)),
    (8440, 3836, 200, 0, 0, (256, 64, 64), (128, 64, 64)),               # more tiles than a round of compute units has
    (200, 8448, 3840, 0, 0, (64, 64, 256), (64, 64, 128)),
    (3848, 136, 8180, 8, 0, (64, 256, 64), (64, 128, 64)),
]


def matrix(g, rows, cols, dtype, pad, shift, by=1.0):
    memory = torch.full((rows * (cols + pad) + shift + 8,), float("nan"), dtype=dtype, device="cuda")
    x = memory.as_strided((rows, cols), (cols + pad, 1), shift)
    return x.copy_(torch.randn((rows, cols), generator=g, device="cuda") * by)


def near(y, e, bound, what):
    off = (y.double() - e).abs()
    bad = ~(off <= bound)
    assert not bad.any(), (what, int(bad.sum()), [tuple(map(int, i)) for i in bad.nonzero()[:3]], float((off / bound).nan_to_num(float("inf")).max()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_larger_tiles(dtype, case):
    M, N, K, pad, shift = CASES[case][:5]
    g = torch.Generator(device="cuda").manual_seed(case)
    x, w = matrix(g, M, K, dtype, pad, shift), matrix(g, N, K, dtype, pad, shift, K ** -0.5)
    bias = (torch.randn(N, generator=g, device="cuda") * 0.3).to(dtype)
    other, dout = matrix(g, M, N, dtype, pad, shift), matrix(g, M, N, dtype, pad, shift)
    d = lambda t: t.double()  # noqa: E731
    for act, b, r in (("gelu", bias, other), (None, None, None)):
        out, z = B.znni_linear(x, w, b, act=act, residual=r, keep=True)
        o, bo, zz, bz = R.linear(d(x), d(w), None if b is None else d(b), act, None if r is None else d(r), dtype)
        near(out, o, bo, f"{act} out")
        near(z, zz, bz, f"{act} z")
        del o, bo, zz, bz
    for act in ("silu", None):
        outs = matrix(g, M, K, dtype, pad, shift), matrix(g, N, K, dtype, pad, shift)
        got = B.znni_linear_backward(dout, x, w, z=None if act is None else other, act=act, dx=outs[0], dw=outs[1])
        for name, y, (e, b) in zip(("dx", "dw", "dbias"), got, R.linear_back(d(dout), d(x), d(w), d(other), act, dtype)):
            near(y, e, b, f"{act} {name}")
        if pad:                                          # what lies between the rows stays as it was
            for y in outs:
                rows, cols = y.shape
                assert torch.isnan(y.as_strided((rows, pad), (cols + pad, 1), shift + cols)).all()


@pytest.mark.parametrize("case", [1, 4, 7])
def test_what_is_not_finite_stays_in_its_row(case):
    """Tiles that end early hold rows again, or zeros, whose products nobody keeps."""
    dtype = torch.bfloat16
    M, N, K, pad, shift = CASES[case][:5]
    g = torch.Generator(device="cuda").manual_seed(100 + case)
    x, w = matrix(g, M, K, dtype, pad, shift), matrix(g, N, K, dtype, pad, shift, K ** -0.5)
    plain = B.znni_linear(x, w)
    x[M - 1, K - 1], x[3, 0] = float("nan"), float("inf")
    got = B.znni_linear(x, w)
    assert torch.equal(got[4:M - 1], plain[4:M - 1]) and torch.equal(got[:3], plain[:3]) and not torch.isfinite(got[[3, M - 1]]).any()
    dx, dw, _ = B.znni_linear_backward(plain, x, w, bias=False)
    assert torch.isfinite(dx).all() and torch.isfinite(dw[:, 1:K - 1]).all() and not torch.isfinite(dw[:, [0, K - 1]]).any()
