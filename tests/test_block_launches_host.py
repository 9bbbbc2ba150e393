"""What calls of products, norms and attention's gradients launch (a recorder stands in for the launches; addresses are made up and never used)."""
import pytest

import launches
from paper_1606_05688_amd import binding as B

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
