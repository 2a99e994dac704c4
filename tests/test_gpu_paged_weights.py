"""Weights of few tokens over a bf16 cache carry more digits than a bf16 number: sums that cancel show them."""
import pytest
import torch

from tests import paged_reference as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nq,nkv,hd", [(16, 8, 128), (8, 1, 64), (40, 2, 128)])
@pytest.mark.parametrize("cached,fresh", [([1, 3, 7], [1, 1, 1]), ([2000], [1]), ([9000, 1], [1, 1])])
def test_single_tokens_over_values_that_cancel(nq, nkv, hd, cached, fresh):
    """Values are 1 and -1 in turn, so a result is the difference of the weights' sums, whose own rounding to bf16 would be 2^-8 of it or
    more.  With two bf16 numbers a weight is right to 2^-16 of it, and the result to twice that beside its own rounding and the bound of fp32."""
    s = R.Step(cached, fresh, 16, nq, nkv, hd, torch.bfloat16, seed=21, stale=float("nan"))
    s.make_plan()
    s.V[:, :, 0::2], s.V[:, :, 1::2] = 1.0, -1.0
    out = s.attend()
    ref, room = R.attend(s.Q, s.K, s.V, s.full_table, s.cached, s.cu, nq, nkv, hd, dtype=torch.float32)
    R.close(out, ref, room + 2 * 2.0 ** -16 + 1.01 * R.HALF_STEP[torch.bfloat16] * ref.abs())
