"""Attention over a cache without pages."""
import pytest
import torch

from paper_1606_05688_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("Lq,max_len", [(1, 60), (3, 60), (1, 50000)])
def test_an_empty_pool_needs_no_table(Lq, max_len):
    """No page is one of none: every row is zero, and neither codes nor a table are read, so that all of them may be NULL."""
    Bn, Hq, Hk, D = 2, 4, 2, 64
    q = torch.randn(Bn * Lq, Hq, D, device=DEV)
    out = torch.full_like(q, float("nan"))
    lens = torch.tensor([60, 7], dtype=torch.int32, device=DEV)
    need = B.znni_kv8_attn_workspace(torch.float32, Bn, Lq, Hq, Hk, D, max_len)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    heads = [B._descriptor(x.data_ptr(), Hq * D, D) for x in (q, out)]
    status = B.lib().znni_kv8_attn(B.F32, Bn, Lq, Hq, Hk, D, heads[0], None, None, None, 0, None, 5, lens.data_ptr(), max_len, B.ALL, 0, 1.0,
                                   heads[1], ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert status == 0 and (out == 0).all()
