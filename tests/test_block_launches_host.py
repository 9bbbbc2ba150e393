"""What calls of products, norms and attention's gradients launch (a recorder stands in for the launches; addresses are made up and never used)."""
import re

import pytest

import launches
from paper_1606_05688_amd import binding as B
from test_gpu_attn_back_single import CASES as SINGLE
from test_gpu_linear_tiles import CASES

P, WS, BIG = 1 << 12, 1 << 20, 1 << 50


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    recorder = launches.make_recorder(tmp_path_factory.mktemp("rec"))
    return lambda calls: launches.record(recorder, B.lib()._name, calls)


def linear_back(type, M, N, K, act, wanted, workspace=WS):
    dx, dw, dbias = (wanted & bit for bit in (B.LINEAR_DX, B.LINEAR_DW, B.LINEAR_DBIAS))
    return ["znni_linear_backward", [["i", type], ["i", M], ["i", N], ["i", K], ["rows", [P, N]], ["rows", [P, K]], ["rows", [P, K]], ["rows", [P, N]], ["i", act],
                                     ["rows", [P, K] if dx else None], ["rows", [P, K] if dw else None], ["p", P if dbias else None], ["p", workspace],
                                     ["z", BIG if workspace else 0], ["p", None]]]


@pytest.mark.parametrize("type", [B.F32, B.BF16, B.F16])
def test_gradients_that_nobody_wants(record, type):
    """A layer whose weights, bias and inputs are all frozen: no workspace, and nothing is launched that would write to one."""
    for status, launched in record([linear_back(type, 8, 16, 64, act, 0, None) for act in range(4)]):
        assert status == 0 and launched == []
    # with an activation, what goes into it is made wherever something is wanted
    for wanted in range(1, 8):
        (status, launched), = record([linear_back(type, 8, 16, 64, 2, wanted)])
        assert status == 0 and "k_slope" in launched[0][0]


def norm(type, T, C, back=False, sums=False):
    if not back:
        return ["znni_block_norm", [["i", type], ["i", T], ["i", C], ["rows", [P, C]], ["rows", [P, C]], ["rows", None], ["p", None], ["p", None], ["f", 1.0], ["f", 1e-5],
                                    ["u", B.NORM_POST | B.NORM_PRE], ["rows", [P, C]], ["rows", [P, C]], ["p", None]]]
    return ["znni_block_norm_backward", [["i", type], ["i", T], ["i", C], ["rows", [P, C]], ["rows", [P, C]], ["rows", [P, C]], ["rows", [P, C]], ["rows", None], ["p", None],
                                         ["p", None], ["f", 1.0], ["f", 1e-5], ["u", B.NORM_POST | B.NORM_PRE], ["rows", [P, C]], ["rows", [P, C]], ["rows", None],
                                         ["p", None], ["p", P if sums else None], ["p", WS], ["z", BIG], ["p", None]]]


@pytest.mark.parametrize("T", [1, 1000, (1 << 22) - 1, 1 << 22, 1 << 23, (1 << 25) + 5, 1 << 30])
def test_a_dimension_of_a_launch_has_fewer_than_2_32_threads(record, T):
    """Many rows of one workgroup each, of up to 1024 threads; every row has its place."""
    cases = [(C, back, sums) for C in (100, 2048, 2049, 4096, 8192, 9000, 16384) for back in (False, True) for sums in ((False, True) if back else (False,))]
    for (C, back, sums), (status, launched) in zip(cases, record([norm(B.BF16, T, *c) for c in cases])):
        assert status == 0 and len(launched) == (2 if sums else 1), (C, back, sums)
        for name, grid, block in launched:
            assert all(g * b < 1 << 32 for g, b in zip(grid, block)) and max(grid[1:]) < 1 << 16, (name, grid, block)
        _, grid, block = launched[0]
        if not sums:
            rows = 4 if block[0] == 256 and C <= (512 if back else 2048) and (back or C <= 512 or T > 1024) else 1
            assert grid[0] * grid[1] * rows >= T, (C, back, grid, block)


@pytest.mark.parametrize("C", [1, 512, 513, 4096, 16384])
def test_workspace_of_sums_over_tokens(record, C):
    """As much as the workgroups leave, and never less for more tokens."""
    import torch
    tokens = [0, 1, 2, 3, 4, 5, 8, 100, 1023, 1024, 1025, 2047, 2048, 2049, 4096, 4097, 1 << 20, 1 << 30]
    sizes = [B.znni_block_norm_backward_workspace(torch.bfloat16, T, C) for T in tokens]
    assert sizes == sorted(sizes) and sizes[0] == 0 and sizes[1] <= 3 * (4 * C + 255) and sizes[-1] <= 3 * 1024 * (4 * C + 255)
    for T, size, (status, launched) in zip(tokens[1:], sizes[1:], record([norm(B.BF16, T, C, True, True) for T in tokens[1:]])):
        name, grid, _ = launched[0]
        assert status == 0 and "k_norm_back" in name and size >= 3 * grid[0] * grid[1] * C * 4


def tile(name):
    """Edge of the tiles of a launch's kernel."""
    if "k_gradients" in name:
        return 64
    waves_n, waves_m, n, m = (int(x) for x in re.search(r"k_productI\w+?Lb[01]ELb[01]ELi(\d)ELi(\d)ELi(\d)ELi(\d)E", name).groups())
    assert waves_n * n == waves_m * m
    return 32 * waves_n * n


@pytest.mark.parametrize("case", range(len(CASES)))
def test_tiles_of_the_cases_that_name_them(record, case):
    M, N, K, pad, shift, small, fp32 = CASES[case]
    for type, kinds in ((B.BF16, small), (B.F16, small), (B.F32, fp32)):
        forward = ["znni_linear", [["i", type], ["i", M], ["i", N], ["i", K], ["rows", [P, K + pad]], ["rows", [P, K + pad]], ["p", None], ["i", 0], ["rows", None], ["rows", None],
                                   ["rows", [P, N + pad]], ["p", WS], ["z", BIG], ["p", None]]]
        calls = [forward, linear_back(type, M, N, K, 0, B.LINEAR_DX), linear_back(type, M, N, K, 0, B.LINEAR_DW)]
        got = record(calls)
        assert [status for status, _ in got] == [0, 0, 0]
        assert tuple(tile(next(n for n, _, _ in launched if "k_product" in n)) for _, launched in got) == kinds
    # each size of tile is there in each form
    for form in range(3):
        assert {c[5][form] for c in CASES} == {64, 128, 256} and 128 in {c[6][form] for c in CASES}


def attention_back(type, case):
    lens, Hq, Hk, D, left, right, sinks = case
    q, k = ["heads", [P, Hq * D, D]], ["heads", [P, Hk * D, D]]
    most = [max(n) for n in zip(*lens)]
    return ["znni_attn_window_backward", [["i", x] for x in (type, len(lens), Hq, Hk, D)] + [q, k, k, q, ["p", P], q, ["p", P], ["p", P]]
            + [["i", x] for x in (*most, left, right, sinks)] + [["f", 1.0], q, k, k, ["p", WS], ["z", BIG], ["p", None]]]


@pytest.mark.parametrize("type", [B.BF16, B.F16])
def test_weights_of_attention_gradients_are_single_where_rows_see_many_keys(record, type):
    got = record([attention_back(type, c) for c in SINGLE])
    assert all(status == 0 for status, _ in got)
    for case, (_, launched) in zip(SINGLE, got):
        assert any(re.search(r"k_backI\w+?Lb0E", name) for name, _, _ in launched), case
    # all widths of heads, dk and dv at once and apart, with a join and without
    assert {(c[3] + 31) // 32 for c in SINGLE} == {1, 2, 3, 4}
    assert {any("k_back_join" in name for name, _, _ in launched) for _, launched in got} == {True, False}
    (_, few), = record([attention_back(type, ([(300, 300)], 2, 1, 64, 100, 0, 0))])
    assert any(re.search(r"k_backI\w+?Lb1E", name) for name, _, _ in few)
