"""The operators on a paged cache beside the framework's others: sequences that share pages, whole sequences, a layer's attention."""
import numpy as np
import pytest
import torch

from paper_2510_15620_amd import binding as B
from tests import paged_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _ints(a):
    return torch.as_tensor(np.asarray(a, np.int32)).to(DEV)


@pytest.mark.parametrize("dtype,nq,nkv,hd", [(F16, 8, 2, 128), (BF16, 14, 2, 64), (F32, 4, 2, 64)])
@pytest.mark.parametrize("prefix,own,fresh", [(3, [0, 5, 40], [1, 1, 1]), (2, [0, 17], [90, 3]), (120, [3, 0, 0], [2, 1, 50])])
def test_sequences_that_share_the_pages_of_a_prefix(dtype, nq, nkv, hd, prefix, own, fresh):
    """Sequences that begin with the same full pages: the same bits as with pages of their own that hold the same, and the shared ones stay as they were."""
    page, n = 16, len(own)
    cached = [prefix * page + x for x in own]
    s = R.Step(cached, fresh, page, nq, nkv, hd, dtype, seed=prefix, stale=float("nan"))
    for i in range(1, n):                                        # the same prefix in every sequence's own pages
        a, b = (torch.as_tensor(s.full_table[j, :prefix], dtype=torch.int64).to(DEV) for j in (i, 0))
        s.K[a], s.V[a] = s.K[b].clone(), s.V[b].clone()
    s.make_plan()
    apart = s.check()
    K, V = s.K.clone(), s.V.clone()
    QKV = torch.randn(s.T, (nq + 2 * nkv) * hd, generator=torch.Generator().manual_seed(1)).to(DEV)
    s.table[:, :prefix] = s.table[0, :prefix]                    # from here on everybody's is the first one's
    shared = s.make_plan()
    want = s.full_table.copy()
    want[:, :prefix] = want[0, :prefix]
    assert np.array_equal(s.d_table.cpu().numpy(), want)
    assert torch.equal(s.check(table=want), apart)
    Q = torch.empty(s.T, nq * hd, dtype=dtype, device=DEV)
    B.op_qkv_finish_paged(QKV, shared["pos"], shared["slot"], s.cache, None, None, 1e-6, 1e6, False, Q)
    kept = torch.as_tensor(want[0, :prefix], dtype=torch.int64).to(DEV)
    assert torch.equal(s.K[kept], K[kept]) and torch.equal(s.V[kept], V[kept])
    s.Q = Q
    s.check(table=want)


@pytest.mark.parametrize("dtype,nq,nkv,hd", [(F16, 16, 8, 128), (BF16, 32, 8, 128), (F32, 4, 2, 64)])
@pytest.mark.parametrize("lens", [[1, 63, 64, 65, 200], [500, 17]])
def test_whole_sequences_as_the_operators_without_a_cache(dtype, nq, nkv, hd, lens):
    """A layer's attention from the normalised rows on, by product, finishing, attention and output product, through pages and without them:
    finished values and attention agree with the same definition, and the layer's results differ by no more than the two attentions may."""
    T, n, page, hidden = sum(lens), len(lens), 16, 256
    g = torch.Generator().manual_seed(T)
    X = torch.randn(T, hidden, generator=g).to(dtype).to(DEV)
    W = (torch.randn((nq + 2 * nkv) * hd, hidden, generator=g) / 16).to(dtype).to(DEV)
    Wo = (torch.randn(hidden, nq * hd, generator=g) / (nq * hd) ** 0.5).to(dtype).to(DEV)
    gains = [(1 + 0.1 * torch.randn(hd, generator=g)).to(dtype).to(DEV) for _ in range(2)]
    QKV = torch.empty(T, (nq + 2 * nkv) * hd, device=DEV)
    store = B.EPI_STORE if dtype == F32 else B.EPI_STORE_F32
    B.op_gemm(store, X, W, QKV)
    # through pages
    s = R.Step([0] * n, lens, page, nq, nkv, hd, dtype, stale=float("nan"))
    d = s.make_plan()
    B.op_qkv_finish_paged(QKV, d["pos"], d["slot"], s.cache, *gains, 1e-6, 1e6, True, s.Q)
    paged = s.check()
    # without: the same rounded queries, keys and values
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    at = d["slot"].long()
    k, v = (t.transpose(1, 2).reshape(-1, nkv * hd)[at] for t in (s.K, s.V))
    plain = torch.empty(T, nq * hd, dtype=dtype, device=DEV)
    if dtype == F32:
        B.op_attention(B.DTYPE_FP32, torch.cat([s.Q, k, v], 1).contiguous(), None, 0, cu, None, nq, nkv, hd, plain)
    else:
        col0 = np.concatenate([[0], np.cumsum([-(-x // 64) * 64 for x in lens])]).astype(np.int32)
        ncol = int(col0[-1])
        col = np.repeat(col0[:-1], lens) + B.vt_column_of_key(d["pos"].cpu().numpy())
        Vt = torch.zeros(nkv, hd, ncol, dtype=F16, device=DEV)
        Vt[:, :, torch.as_tensor(col, dtype=torch.int64).to(DEV)] = v.view(T, nkv, hd).permute(1, 2, 0).to(F16)
        B.op_attention(B._dt(s.Q), torch.cat([s.Q, k], 1).contiguous(), Vt, ncol, cu, col0[:-1].copy(), nq, nkv, hd, plain)
    ref, room = R.attend(s.Q, s.K, s.V, s.full_table, s.cached, s.cu, nq, nkv, hd, dtype=dtype)
    R.close(plain, ref, room)
    out = [torch.empty(T, hidden, device=DEV) for _ in range(2)]
    for o, a in zip(out, (paged, plain)):
        B.op_gemm(store, a, Wo, o)
    # both attentions are within `room` of the definition; the products' fp32 sums of nq hd terms are off by 2^-24 (nq hd + 1) of the magnitudes
    w = Wo.double().cpu().abs()
    most = 2 * room @ w.T + 2 * (nq * hd + 1) * 2.0 ** -24 * ((ref.abs() + room) @ w.T)
    assert ((out[0] - out[1]).double().cpu().abs() <= most).all()
