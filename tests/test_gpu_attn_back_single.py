"""Gradients of windowed attention where rows see many keys and weights of 16-bit types are single values: windows, first tokens, ragged and empty
sequences, walks that are split, what is not finite.  Which weights a case takes is checked without a GPU (test_block_launches_host.py)."""
import pytest
import torch

import test_gpu_attn_back as T
from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
ALL = B.ALL

CASES = [
    ([(900, 900)], 4, 2, 64, 560, 0, 0),
    ([(700, 1400), (33, 600), (0, 9), (7, 0), (600, 20)], 2, 1, 128, 520, 0, 4),
    ([(1300, 1300)], 2, 2, 40, 300, 250, 3),
    ([(1100, 1100), (1, 530)], 3, 1, 96, 510, 2, 0),
    ([(1000, 1000)], 2, 1, 128, 600, 0, 40),                    # first tokens' rows past the window, in heads whose dk and dv are apart
    ([(1500, 1500)], 1, 1, 32, 512, 0, 600),                    # more first tokens than a tile has keys, and than the window
    ([(5, 3000)], 8, 2, 72, 2000, 0, 2),                        # the walk over the keys is split
    ([(2000, 600)], 2, 1, 112, 530, ALL, 0),                    # the walk over the rows is split, early rows see nothing on their left
    ([(600, 600)], 48, 3, 88, ALL, 0, 0),
    ([(777, 640)], 2, 2, 16, 600, 5, 1),                        # the first rows see nothing
    ([(600, 600)], 64, 64, 40, 520, 0, 0),                      # enough workgroups: no walk is split
    ([(1100, 1100)], 32, 32, 72, 600, 0, 3),
    ([(1030, 1030)], 64, 32, 128, 540, 0, 0),
]


@pytest.fixture(autouse=True)
def these_cases(monkeypatch):
    monkeypatch.setattr(T, "CASES", CASES)


@pytest.mark.parametrize("dtype", T.TYPES)
@pytest.mark.parametrize("case", range(len(CASES)))
def test_cases(dtype, case):
    T.test_cases(dtype, case)


@pytest.mark.parametrize("dtype", T.TYPES)
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("case", [0, 2, 4, 5])
def test_not_finite(dtype, bad, case):
    T.test_not_finite(dtype, bad, case)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_strides_and_runs(dtype):
    """Heads of tokens that lie apart, and the same call again: the same bits."""
    lens, Hq, Hk, D, left, right, sinks = CASES[1]
    (q, k, v, dout), where = T.make(lens, Hq, Hk, D, dtype, 31)
    out, stats, got = T.call((q, k, v, dout), where, left, right, sinks)
    wide = lambda x: torch.full((x.shape[0], x.shape[1] + 1, D + 8), float("nan"), dtype=dtype, device="cuda")[:, 1:, 8:].copy_(x)  # noqa: E731
    for form in (torch.clone, wide):
        a, b, c, e, o = (form(x) for x in (q, k, v, dout, out))
        outs = [form(torch.zeros_like(x)) for x in (q, k, v)]
        again = B.znni_attn_window_backward(e, a, b, c, o, stats, *where, left=left, right=right, sinks=sinks, dq=outs[0], dk=outs[1], dv=outs[2])
        assert all(torch.equal(x, y) for x, y in zip(again, got))
