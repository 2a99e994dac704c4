"""Score caps from far below the scores to far above them, against 64 bits, with a bound that does not grow with the cap."""
import math

import pytest
import torch

from tests import paged_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _room(s, ref, scale, slopes):
    """How far a result may be from `ref`: the bound for the same scores without a cap (R.attend has it), which holds with one too, since a
    capped score and its change with the score are no larger than without.  For the result's own rounding `ref` counts."""
    plain, room = R.attend(s.Q, s.K, s.V, s.full_table, s.cached, s.cu, s.nq, s.nkv, s.hd, scale, 0.0, s.window, slopes, s.dtype)
    return room + 1.01 * R.HALF_STEP[s.dtype] * (ref - plain).abs()


@pytest.mark.parametrize("dtype,nq,nkv,hd", [(F16, 8, 2, 128), (F16, 6, 2, 64), (BF16, 8, 2, 128), (F32, 4, 2, 64)])
@pytest.mark.parametrize("cached,fresh", [([300], [1]), ([100, 30], [5, 1]), ([200], [90])])
@pytest.mark.parametrize("cap,scale", [(1e3, 0.0), (1e4, 0.0), (1e5, 0.0), (1e6, 0.0), (1e8, 0.0), (1e30, 0.0), (9e36, 0.0), (30.0, 0.0), (10.0, 1.0),
                                       (20.0, 1.0), (40.0, 1.0), (64.0, 1.0), (64.5, 1.0), (80.0, 1.0), (1.0, 0.0), (1e-3, 0.0), (1e-30, 0.0)])
def test_caps_of_every_size(dtype, nq, nkv, hd, cached, fresh, cap, scale):
    """Caps at which every score is small against the cap, at which some are (scale 1: scores of some 10), and which all scores reach."""
    s = R.Step(cached, fresh, 16, nq, nkv, hd, dtype, seed=12, stale=float("nan"))
    s.make_plan()
    slopes = torch.exp2(-8.0 * torch.arange(1, nq + 1) / nq).to(DEV) if fresh[0] == 5 else None
    ref, _ = R.attend(s.Q, s.K, s.V, s.full_table, s.cached, s.cu, nq, nkv, hd, scale, cap, 0, slopes, dtype)
    R.close(s.attend(scale, cap, slopes)[: s.cu[-1]], ref, _room(s, ref, scale, slopes))


@pytest.mark.parametrize("dtype,nq,nkv,hd", [(F16, 8, 2, 128), (BF16, 14, 2, 64), (F32, 4, 2, 64)])
@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("cap,scale", [(100.0, 2.0), (1e5, 0.0), (1e20, 1.0)])
def test_large_caps_with_slopes_windows_and_missing_pages(dtype, nq, nkv, hd, window, cap, scale):
    s = R.Step([150, 20], [60, 1], 16, nq, nkv, hd, dtype, seed=14, window=window, stale=float("nan"))
    s.make_plan()
    s.full_table[0, 7] = -1
    s.d_table = s.device(s.full_table)
    slopes = torch.exp2(-8.0 * torch.arange(1, nq + 1) / nq).to(DEV)
    ref, _ = R.attend(s.Q, s.K, s.V, s.full_table, s.cached, s.cu, nq, nkv, hd, scale, cap, window, slopes, dtype)
    R.close(s.attend(scale, cap, slopes)[: s.cu[-1]], ref, _room(s, ref, scale, slopes))


@pytest.mark.parametrize("dtype,hd", [(F16, 128), (F16, 64), (BF16, 128), (F32, 64)])
@pytest.mark.parametrize("fresh", [1, 40])
@pytest.mark.parametrize("cap,factor", [(1e4, 1e3), (1e5, 1e4), (1e5, 2e3)])
def test_small_scores_beside_one_that_reaches_the_cap(dtype, hd, fresh, cap, factor):
    """Key 0's score is minus `factor` times a query's square, near or beyond minus the cap: it has no weight, and the others keep their digits."""
    nq = nkv = 2
    s = R.Step([60], [fresh], 16, nq, nkv, hd, dtype, seed=13, stale=float("nan"))
    s.make_plan()
    s.Q.copy_(s.Q[:1].expand_as(s.Q).clone())                     # one query for all rows, so that key 0 meets all of them alike
    pg = int(s.full_table[0, 0])
    s.K[pg, :, 0] = (-factor * s.Q[0].view(nq, hd).float()).to(dtype)
    got = s.attend(0.0, cap).view(fresh, nq, hd).double().cpu()
    key = torch.arange(60 + fresh)
    pages = torch.as_tensor(s.full_table[0], dtype=torch.int64)[key // 16]
    K, V, Q = s.K.double().cpu()[pages, :, key % 16], s.V.double().cpu()[pages, :, key % 16], s.Q.double().cpu().view(fresh, nq, hd)
    for h in range(nq):
        x = K[:, h] @ Q[0, h] / math.sqrt(hd)
        x = cap * torch.tanh(x / cap)
        assert x[0] < -2000
        for i in range(fresh):
            n = 61 + i
            w = torch.softmax(x[:n], 0)
            want, big = w @ V[:n, h], V[:n, h].abs().max()
            # errors of the scores that have weight, in the sums and the steps behind them (as R.attend has them), of the weights and the sums over n
            e = (hd + 2) * 2.0 ** -24 * (K[1:n, h].abs() @ Q[0, h].abs()).max() / math.sqrt(hd) + x[1:n].abs().max() * 2.0 ** -20 + n * 2.0 ** -24
            e += R.HALF_STEP[dtype] if dtype != F32 else 2.0 ** -22
            room = 2.1 * e * big + 1.01 * R.HALF_STEP[dtype] * want.abs() + (2.0 ** -25 if dtype == F16 else 0.0)
            assert ((got[i, h] - want).abs() <= room).all(), (h, i, float((got[i, h] - want).abs().max()), float(room.max()))
