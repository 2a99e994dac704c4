"""A whole layer whose products run on 8-bit integers, over a paged cache: norm, q/k/v product, finishing, attention, codes of its results, O product into the stream, then the
feed-forward block.  Every operator against its own definition in 64 bits, on what the one before it left."""
import numpy as np
import pytest
import torch

from paper_2510_15620_amd import binding as B
from tests import paged_reference as R
from tests import test_gpu_q8 as Q

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


class Layer:
    def __init__(self, hidden, ffn, nq, nkv, hd, dtype, rows, seed):
        g = torch.Generator().manual_seed(seed)
        self.hidden, self.ffn, self.nq, self.nkv, self.hd, self.dtype = hidden, ffn, nq, nkv, hd, dtype

        def weights(n, k):
            q = B.Q8(n, k)
            B.op_quantize_q8((torch.randn(n, k, generator=g) / k ** 0.5).to(BF16).cuda(), q)
            return q
        self.Wqkv, self.Wo, self.W1, self.W2 = weights((nq + 2 * nkv) * hd, hidden), weights(hidden, nq * hd), weights(2 * ffn, hidden), weights(hidden, ffn)
        self.norm1, self.norm2 = ((1 + 0.1 * torch.randn(hidden, generator=g)).to(BF16).cuda() for _ in range(2))
        self.q_gain, self.k_gain = ((1 + 0.1 * torch.randn(hd, generator=g)).to(dtype).cuda() for _ in range(2))
        # activations, for the largest step
        self.x8, self.o8, self.h8 = B.Q8(rows, hidden), B.Q8(rows, nq * hd), B.Q8(rows, ffn)

    def buffers(self, T):
        empty = lambda n, dtype: torch.empty(T, n, dtype=dtype, device="cuda")  # noqa: E731
        return {"QKV": empty((self.nq + 2 * self.nkv) * self.hd, F32), "Q": empty(self.nq * self.hd, self.dtype), "out": empty(self.nq * self.hd, self.dtype),
                "h": empty(self.ffn, self.dtype), "x8": self.x8.first(T), "o8": self.o8.first(T), "h8": self.h8.first(T)}

    def attention(self, X, b, plan, pos, slot, cache, table, work):
        B.op_rmsnorm_q8(X, self.norm1, 1e-6, b["x8"])
        B.op_gemm_q8(B.EPI_STORE_F32, b["x8"], self.Wqkv, b["QKV"])
        B.op_qkv_finish_paged(b["QKV"], pos, slot, cache, self.q_gain, self.k_gain, 1e-6, 1e6, True, b["Q"])
        B.op_attention_paged(plan, b["Q"], cache, table, b["out"], work)
        B.op_quantize_q8(b["out"], b["o8"])
        B.op_gemm_q8(B.EPI_RESIDUAL, b["o8"], self.Wo, X)

    def feed_forward(self, X, b):
        B.op_rmsnorm_q8(X, self.norm2, 1e-6, b["x8"])
        B.op_gemm_q8(B.EPI_SWIGLU, b["x8"], self.W1, b["h"])
        B.op_quantize_q8(b["h"], b["h8"])
        B.op_gemm_q8(B.EPI_RESIDUAL, b["h8"], self.W2, X)


def codes(q):
    return q.codes[:, :q.cols]


def ints(a):
    return torch.as_tensor(np.asarray(a, np.int32)).cuda()


def check_codes(x, q):
    want, _ = Q.exact_codes(Q.host(x))
    assert torch.equal(Q.codes_of(q), torch.round(want))
    Q.check_padding(q)


@pytest.mark.parametrize("hidden,ffn,nq,nkv,hd,dtype", [(512, 1408, 8, 2, 128, F16), (1003, 1500, 5, 1, 64, BF16)])
def test_a_layer_over_a_paged_cache(hidden, ffn, nq, nkv, hd, dtype):
    """Two sequences: one read in chunks and then single tokens, one that joins late; a step of one token, of a sequence without any."""
    n_pages, page, width = 40, 16, 25
    layer = Layer(hidden, ffn, nq, nkv, hd, dtype, 131, seed=hidden)
    g = torch.Generator().manual_seed(ffn)
    K, V = (torch.full((n_pages, nkv, page, hd), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    cache, table = B.KVCache(K, V), ints(np.full((2, width), -1))
    free, n_free = ints(np.random.default_rng(1).permutation(n_pages)), ints([n_pages])
    cached = np.zeros(2, np.int32)
    for fresh in ([130, 1], [1, 1], [0, 47], [1, 0], [3, 120]):
        T = sum(fresh)
        plan = B.PagePlan(2, T, nq, nkv, page, n_pages, width)
        cu, pos, slot, status = ints([0] * 3), ints([0] * T), ints([0] * T), ints([0] * 4)
        B.op_page_plan(plan, ints(cached), ints(fresh), table, free, n_free, n_free, cu, pos, slot, status)
        X = (torch.randn(T, hidden, generator=g) * torch.exp(torch.randn(T, 1, generator=g))).cuda()
        b, before, old = layer.buffers(T), X.clone(), (K.double().cpu(), V.double().cpu())
        layer.attention(X, b, plan, pos, slot, cache, table, B.attention_paged_workspace(plan, cache))
        assert status.tolist() == [T, status.tolist()[1], 0, 0]
        Q.check_norm(before.cpu(), None, layer.norm1.cpu(), 1e-6, b["x8"], before.cpu())
        Q.check_product(B.EPI_STORE_F32, F32, b["QKV"], None, Q.product(codes(b["x8"]), b["x8"].scales, codes(layer.Wqkv), layer.Wqkv.scales))
        want = R.finish(b["QKV"].double().cpu(), pos.cpu(), slot.cpu(), *old, layer.q_gain.double().cpu(), layer.k_gain.double().cpu(), 1e-6, 1e6, nq, nkv, hd)
        for got, ref in zip((b["Q"], K, V), want):
            R.close(got, ref, ref.abs() * R.HALF_STEP[dtype] * 1.01 + 2.0 ** -24 * (hd / 2 + 12) * 3 * ref.abs().nan_to_num(0.0).max())
        ref, room = R.attend(b["Q"], K, V, table.cpu().numpy(), cached, cu.cpu().numpy(), nq, nkv, hd, dtype=dtype)
        R.close(b["out"], ref, room)
        check_codes(b["out"], b["o8"])
        Q.check_product(B.EPI_RESIDUAL, F32, X, before, Q.product(codes(b["o8"]), b["o8"].scales, codes(layer.Wo), layer.Wo.scales))
        before = X.clone()
        layer.feed_forward(X, b)
        Q.check_norm(before.cpu(), None, layer.norm2.cpu(), 1e-6, b["x8"], before.cpu())
        Q.check_product(B.EPI_SWIGLU, dtype, b["h"], None, Q.product(codes(b["x8"]), b["x8"].scales, codes(layer.W1), layer.W1.scales))
        check_codes(b["h"], b["h8"])
        Q.check_product(B.EPI_RESIDUAL, F32, X, before, Q.product(codes(b["h8"]), b["h8"].scales, codes(layer.W2), layer.W2.scales))
        cached = cached + np.array(fresh, np.int32)


def test_a_layer_captured_and_replayed():
    """Single tokens of 24 sequences: the layer in a graph, replayed on other streams of numbers with eager work between, has the eager calls' bits each time."""
    n, page, width, n_pages, nq, nkv, hd = 24, 16, 8, 24 * 8, 8, 2, 128
    layer = Layer(512, 1408, nq, nkv, hd, F16, n, seed=3)
    r, lens = np.random.default_rng(2), np.random.default_rng(3).integers(0, width * page - 1, n)
    g = torch.Generator(device="cuda").manual_seed(4)
    pool = [torch.randn(n_pages, nkv, page, hd, generator=g, device="cuda").half() for _ in range(2)]
    pages = ints(r.permutation(n_pages).reshape(n, width))
    sides = []
    for _ in range(2):
        s = {"K": pool[0].clone(), "V": pool[1].clone(), "X": torch.zeros(n, 512, device="cuda"), "table": pages.clone()}
        s["cache"], s["plan"] = B.KVCache(s["K"], s["V"]), B.PagePlan(n, n, nq, nkv, page, n_pages, width)
        s["cu"], s["pos"], s["slot"] = ints([0] * (n + 1)), ints([0] * n), ints([0] * n)
        s["work"] = B.attention_paged_workspace(s["plan"], s["cache"])
        # no page is taken where the new token's page is there already
        B.op_page_plan(s["plan"], ints(lens), ints([1] * n), s["table"], ints([0]), ints([0]), ints([0]), s["cu"], s["pos"], s["slot"], ints([0] * 4))
        s["table"].copy_(pages)
        s["slot"].copy_(torch.gather(pages, 1, s["pos"][:, None].long() // page)[:, 0] * page + s["pos"] % page)
        sides.append(s)
    eager, graphed = sides
    other = Layer(512, 1408, nq, nkv, hd, F16, n, seed=3)

    def step(s, l, b):
        l.attention(s["X"], b, s["plan"], s["pos"], s["slot"], s["cache"], s["table"], s["work"])
        l.feed_forward(s["X"], b)
    be, bg = layer.buffers(n), other.buffers(n)
    step(eager, layer, be)
    step(graphed, other, bg)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed, other, bg)
    for turn in range(4):
        x = torch.randn(n, 512, generator=g, device="cuda") * (turn + 1)
        eager["X"].copy_(x)
        graphed["X"].copy_(x)
        step(eager, layer, be)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(eager["X"], graphed["X"]) and torch.equal(eager["K"], graphed["K"]) and torch.equal(be["h8"].codes, bg["h8"].codes), turn
        assert torch.isfinite(eager["X"]).all()
