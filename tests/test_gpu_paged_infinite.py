"""Cached values that are not finite, seen with weights that 32 bits do not hold: the result is the same wherever tiles and parts end."""
import pytest
import torch

from tests import paged_reference as R

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dtype,hd", [(F16, 128), (F16, 64), (BF16, 128), (F32, 32), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("cached,fresh,window,at,low", [
    (200, 1, 0, 100, (100, 101)),          # in a tile without a mask
    (200, 1, 0, 10, (0, 64)),              # before all keys that have weight
    (200, 1, 150, 55, (0, 64)),            # at the window's edge, before the others
    (200, 1, 0, 199, (199, 200)),          # in the last tile, which has a mask
    (200, 5, 0, 201, (201, 202)),          # not seen by the first row
    (130, 90, 0, 100, (100, 101)), (130, 90, 0, 20, (0, 64)), (130, 90, 0, 175, (175, 176)), (130, 90, 100, 60, (0, 64)),
    (9000, 1, 0, 4100, (4096, 4608)),      # all keys of a part
    (9000, 3, 0, 100, (100, 101)), (9000, 40, 0, 100, (0, 2048))])
def test_values_that_are_not_finite_whatever_their_weight(dtype, hd, cached, fresh, window, at, low):
    """Scores are 0, of the keys low[0] .. low[1] - 1 -400, a weight of 10^-174 of the others'.  Key `at` has an infinity, a NaN, and beside one of
    another key and the other sign another infinity: a row that sees it has that infinity, NaN and NaN, every other value is as it was."""
    nq, nkv = 8, 2
    s = R.Step([cached], [fresh], 64, nq, nkv, hd, dtype, seed=5, window=window, stale=NAN)
    s.make_plan()
    s.Q.fill_(1.0)
    p = torch.arange(cached + fresh)
    pages = torch.as_tensor(s.full_table[0], dtype=torch.int64)[p // 64].to(s.K.device)
    k = torch.zeros(cached + fresh, device=s.K.device)
    k[low[0]: low[1]] = -400.0 / hd ** 0.5
    s.K[pages, :, (p % 64).to(s.K.device)] = k.to(dtype)[:, None, None].expand(-1, nkv, hd)
    where = lambda i: (int(s.full_table[0, i // 64]), 1, i % 64)  # noqa: E731
    other = cached - 1 if at != cached - 1 else cached - 2
    for i, d in ((at, 3), (at, 9), (at, 20), (at, 21), (other, 20)):
        s.V[where(i)][d] = 1.0
    before = s.attend().view(s.T, nq, hd)
    s.V[where(at)][3], s.V[where(at)][9], s.V[where(at)][20], s.V[where(at)][21] = INF, NAN, INF, -INF
    s.V[where(other)][20] = -INF
    got = s.attend().view(s.T, nq, hd)
    want = before.clone()
    top = 65504.0 if dtype == F16 else INF                       # half results saturate
    for i in range(fresh):
        pos = cached + i
        sees = lambda key: key <= pos and (not window or key > pos - window)  # noqa: E731
        if sees(at):
            want[i, 4:, 3], want[i, 4:, 9], want[i, 4:, 21] = top, NAN, -top
        if sees(at) or sees(other):
            want[i, 4:, 20] = NAN if sees(at) and sees(other) else top if sees(at) else -top
    assert torch.equal(torch.isnan(got), torch.isnan(want)), torch.isnan(got).ne(torch.isnan(want)).nonzero()[:4].tolist()
    assert torch.equal(got.nan_to_num(12345.0, INF, -INF), want.nan_to_num(12345.0, INF, -INF)), got.nan_to_num(12345.0, INF, -INF).ne(want.nan_to_num(12345.0, INF, -INF)).nonzero()[:4].tolist()


@pytest.mark.parametrize("dtype,hd", [(F16, 128), (BF16, 64), (F32, 64)])
@pytest.mark.parametrize("softcap", [0.0, 30.0, 1000.0])
@pytest.mark.parametrize("cached,fresh,at", [(300, 1, 5), (9000, 1, 5), (300, 90, 5), (300, 90, 340), (9000, 40, 8000)])
def test_a_key_whose_values_all_are_nan(dtype, hd, cached, fresh, at, softcap):
    """Rows that see it are NaN in all dimensions of its head, the others keep their bits."""
    s = R.Step([cached], [fresh], 16, 8, 2, hd, dtype, seed=6, stale=NAN)
    s.make_plan()
    s.K[int(s.full_table[0, at // 16]), 0, at % 16] = 0.0
    before = s.attend(softcap=softcap).view(s.T, 8, hd)
    s.V[int(s.full_table[0, at // 16]), 0, at % 16] = NAN
    got = s.attend(softcap=softcap).view(s.T, 8, hd)
    sees = torch.arange(cached, cached + fresh, device=got.device) >= at
    assert torch.isnan(got[sees, :4]).all() and torch.equal(got[~sees], before[~sees]) and torch.equal(got[:, 4:], before[:, 4:])
