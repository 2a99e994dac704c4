"""Attention over a paged cache where scores are no numbers: a query that is NaN, and keys that are NaN and all that a wave or a part sees."""
import pytest
import torch

from tests import paged_reference as R

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN = float("nan")
TYPES = [(F16, 64), (F16, 128), (BF16, 128), (F32, 32), (F32, 64), (F32, 128)]


def _check(s, before, nan, softcap=0.0):
    """`nan` [rows, heads]: there all values are NaN, elsewhere the result has the bits that it had before."""
    got, before, nan = s.attend(softcap=softcap).view(s.T, s.nq, s.hd), before.view(s.T, s.nq, s.hd), nan.to(before.device)
    assert torch.isnan(got[nan]).all(), "a seen NaN was lost"
    assert torch.equal(got[~nan], before[~nan])


@pytest.mark.parametrize("dtype,hd", TYPES)
@pytest.mark.parametrize("softcap", [0.0, 20.0])
@pytest.mark.parametrize("cached,fresh,cut", [([20], [1], False), ([70, 3], [40, 1], False), ([9000, 40], [1, 2], True), ([9000], [40], True)])
def test_a_query_that_is_nan(dtype, hd, cached, fresh, cut, softcap):
    s = R.Step(cached, fresh, 64, 8, 2, hd, dtype, seed=3, pad=1, stale=NAN)
    s.make_plan()
    assert (int(s.plan.buffer[:64].view(torch.int32)[10]) > 0) == cut
    before = s.attend(softcap=softcap)
    assert torch.isfinite(before).all()
    nan = torch.zeros(s.T, s.nq, dtype=torch.bool)
    for row, head in ((0, 1), (fresh[0] - 1, 6)):
        s.Q[row, head * hd + 3] = NAN
        nan[row, head] = True
    _check(s, before, nan, softcap)


@pytest.mark.parametrize("dtype,hd", TYPES)
@pytest.mark.parametrize("cached,fresh,window,first,last", [
    (16, 1, 0, 16, 17), (0, 1, 0, 0, 1), (40, 1, 9, 40, 41),     # one key, alone in its wave's keys, or all that there is
    (0, 90, 1, 60, 61),                                            # every row sees itself only
    (9000, 1, 0, 4096, 4608), (9000, 3, 0, 8992, 9001), (9000, 40, 0, 2048, 4096)])   # all of several runs of tiles, of the last one
def test_keys_that_are_nan(dtype, hd, cached, fresh, window, first, last):
    """Keys first .. last - 1 of KV head 0 are NaN: rows of its query heads that see one are NaN, all others are as before."""
    s = R.Step([cached], [fresh], 64, 8, 2, hd, dtype, seed=4, window=window, stale=NAN)
    s.make_plan()
    before = s.attend()
    for p in range(first, last):
        s.K[int(s.full_table[0, p // 64]), 0, p % 64, 1] = NAN
    pos = torch.arange(cached, cached + fresh)
    sees = pos >= first
    if window:
        sees &= pos - window < last - 1
    nan = torch.zeros(s.T, s.nq, dtype=torch.bool)
    nan[:, : 4] = sees[:, None]
    _check(s, before, nan)
