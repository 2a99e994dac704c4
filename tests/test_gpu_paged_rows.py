"""Every row of a chunk gets its own result, whole: lanes exchange rows on the way to memory."""
import pytest
import torch

from paper_2510_15620_amd import binding as B
from tests import paged_reference as R

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype,hd", [(F16, 64), (F16, 128), (BF16, 64), (BF16, 128), (F32, 32), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("nq,nkv", [(2, 2), (4, 2), (8, 2), (7, 1), (24, 1)])
@pytest.mark.parametrize("cached,fresh", [([5, 0], [1, 33]), ([40], [129]), ([0, 0, 7], [64, 31, 95])])
def test_rows_that_see_themselves_only(dtype, hd, nq, nkv, cached, fresh):
    """With a window of one token a weight is 1, and a result is that token's value of the row's KV head, bit for bit."""
    s = R.Step(cached, fresh, 32, nq, nkv, hd, dtype, seed=hd, pad=2, window=1, stale=float("nan"))
    d = s.make_plan()
    wide = torch.full((s.T, nq * hd + 2 * hd), 7.0, dtype=dtype, device="cuda")
    B.op_attention_paged(s.plan, s.Q, s.cache, s.d_table, wide[:, : nq * hd], B.attention_paged_workspace(s.plan, s.cache))
    n = sum(fresh)
    slot = d["slot"][:n].long()
    v = s.V[slot // 32, :, slot % 32]                            # [rows, KV heads, hd]
    assert torch.equal(wide[:n, : nq * hd].view(n, nkv, nq // nkv, hd), v[:, :, None].expand(n, nkv, nq // nkv, hd))
    assert (wide[n:] == 7).all() and (wide[:, nq * hd:] == 7).all()
