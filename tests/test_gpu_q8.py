"""Operators on 8-bit rows against plain forms in 64 bits.  u = 2^-24, half a step of fp32; each rounding counts one, to 16 bits finfo.eps / 2."""
import itertools

import numpy as np
import pytest
import torch

from paper_2510_15620_amd import binding as B

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
TINY = 2.0 ** -119


def gen(seed):
    return torch.Generator().manual_seed(seed)


def host(t):
    return t.detach().to("cpu").double()


def half_step(dtype):
    return torch.finfo(dtype).eps / 2 if dtype is not F32 else 0.0      # fp32's own rounding is among the counted ones


def smallest(dtype):
    return {F32: 2.0 ** -150, BF16: 2.0 ** -134, F16: 2.0 ** -25}[dtype]     # half of the least subnormal


def codes_of(q):
    return q.codes[:, :q.cols].to("cpu").double()


def check_padding(q):
    assert not q.codes[:, q.cols:].any(), "codes behind a row's end"


def exact_codes(x):
    """Codes (before rounding), scales of finite rows, in 64 bits."""
    top = x.abs().amax(1, keepdim=True)
    return torch.where(top >= TINY, x * 127.0 / top, torch.zeros(())), torch.where(top >= TINY, top / 127.0, torch.zeros(()))[:, 0]


# ------------------------------------------------------------------------------------------------------------------ rows to codes

WIDTHS = [1, 3, 64, 127, 128, 129, 256, 500, 1003, 1024, 1025, 2047, 4096, 4100, 8191, 12288, 16384, 16392, 40001, 131071]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", WIDTHS)
def test_quantize(cols, dtype):
    """16-bit rows: the codes are the nearest integers, ties to even.  fp32: 127 / max and its product with x are rounded (2 u of 127), so
    a code is within half a step and that of x / scale.  The scale is max / 127 rounded once."""
    g = gen(cols)
    x = (torch.randn(9, cols, generator=g) * torch.randn(9, cols, generator=g)).to(dtype)
    x[3] = 0
    x[4] *= 1e-4
    x[5, cols // 2] = 30.0
    x[6, -1] = -float(x[6].abs().max()) * 2                     # half the maximum is a tie: 63.5
    x[6, 0] = x[6, -1] / 2 if cols > 1 else x[6, 0]
    q = B.Q8(9, cols)
    q.codes.fill_(55)
    B.op_quantize_q8(x.cuda(), q)
    want, scale = exact_codes(x.double())
    assert torch.equal(q.scales.cpu(), (x.float().abs().amax(1) / torch.tensor(127.0)))
    if dtype is F32:
        assert (codes_of(q) - want).abs().max() <= 0.5 + 127 * 2.01 * U
    else:
        assert torch.equal(codes_of(q), torch.round(want))
    check_padding(q)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_quantize_every_quotient_of_few_bits(dtype):
    """Rows whose maximum is m (256 values over a factor of two) with every 16-bit number up to it that gives a code of at least 1/4: ties among them."""
    bits = torch.arange(0, 32768, dtype=torch.int32).to(torch.int16).view(dtype)
    bits = bits[torch.isfinite(bits) & (bits > 0)]
    bits = bits[(bits.double() >= 2.0 ** -10) & (bits.double() <= 2.0)]
    tops = bits[(bits.double() >= 1.0) & (bits.double() < 2.0)][:: 1 if dtype is BF16 else 4]
    x = bits[None].repeat(len(tops), 1)
    x = torch.where(x.double() <= tops.double()[:, None], x, -tops[:, None])
    q = B.Q8(*x.shape)
    B.op_quantize_q8(x.cuda(), q)
    xd, td = x.cuda().double(), tops.cuda().double()[:, None]
    assert torch.equal(q.codes[:, :q.cols].double(), torch.round(xd * 127.0 / td))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_extremes(dtype):
    """Infinities and NaN anywhere in a row: scale NaN, codes 0; magnitudes below 2^-119: zeros; the largest numbers keep their codes; other rows do not notice."""
    big = torch.finfo(dtype).max
    x = torch.randn(12, 300, generator=gen(1)).to(dtype)
    x[1, 299] = float("inf")
    x[2, 0] = -float("inf")
    x[3, 128] = float("nan")
    x[4], x[5] = big, -big
    x[5, 7] = big / 2
    x[6] = float("nan")
    x[7] = 0.0
    if dtype is not F16:
        x[8] = 2.0 ** -120
        x[9] = 2.0 ** -119
        x[9, 1] = 2.0 ** -126
    x[10] = -0.0
    q = B.Q8(12, 300)
    B.op_quantize_q8(x.cuda(), q)
    s, c = q.scales.cpu(), codes_of(q)
    bad = torch.zeros(12, dtype=torch.bool)
    bad[[1, 2, 3, 6]] = True
    assert torch.equal(torch.isnan(s), bad) and not c[bad].any()
    want, _ = exact_codes(x[~bad].double())
    top = x[~bad].float().abs().amax(1)
    assert torch.equal(s[~bad], torch.where(top.double() >= TINY, top / torch.tensor(127.0), torch.zeros(())))
    assert (c[~bad] - want).abs().max() <= (0.5 + 127 * 2.01 * U if dtype is F32 else 0.5)
    assert (c[4] == 127).all() and c[5, 7] == 64 and c[5, 8] == -127


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [5, 129, 1003, 2056])
def test_quantize_strides_and_neighbours(cols, dtype):
    """Rows that begin at any value of a larger buffer, codes in the middle of one: nothing beside them is written."""
    buf = torch.randn(20, cols + 9, generator=gen(2)).to(dtype).cuda()
    x = buf[3:16, 1:1 + cols]
    store = torch.full((15, 4096 if cols > 2000 else 2048), 77, dtype=torch.int8, device="cuda")
    q = B.Q8(13, cols)
    q._set(store[1:14], torch.empty(13, device="cuda"), cols)
    B.op_quantize_q8(x, q)
    dense = B.Q8(13, cols)
    B.op_quantize_q8(x.contiguous(), dense)
    w = dense.codes.shape[1]
    assert torch.equal(store[1:14, :w], dense.codes) and torch.equal(q.scales, dense.scales)
    assert (store[0] == 77).all() and (store[14] == 77).all() and (store[1:14, w:] == 77).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 7, 64, 130, 1003, 2048, 5000, 70001])
def test_dequantize(cols, dtype):
    """code * scale rounded to fp32, then to 16 bits: equal bits.  Gaps between the rows stay."""
    g = gen(cols)
    codes = torch.randint(-128, 128, (11, cols), generator=g, dtype=torch.int8)
    scales = torch.rand(11, generator=g) * 10.0 ** torch.randint(-4, 3, (11,), generator=g)
    scales[2], scales[3] = 0.0, float("nan")
    q = B.Q8.of(codes.cuda(), scales.cuda())
    out = torch.full((11, cols + 5), 9.0, dtype=dtype, device="cuda")
    B.op_dequantize_q8(q, out[:, 2:2 + cols])
    want = codes.float() * scales[:, None]
    if dtype is F16:
        want = want.clamp(-65504, 65504)
    assert torch.equal(out[:, 2:2 + cols].cpu().nan_to_num(7.5), want.to(dtype).nan_to_num(7.5)) and torch.isnan(out[3, 2:2 + cols]).all()
    assert (out[:, :2] == 9).all() and (out[:, 2 + cols:] == 9).all()


# ------------------------------------------------------------------------------------------------------------------ norm

def check_norm(x, d, gain, eps, q, got_x):
    """x: what the stream held (fp32, host).  The stream is fl(x + d) to the bit.  p = x gain, its maximum, 127 / max and the product of both are rounded: 4 u of 127 around the
    half step.  The scale: a sum of squares, of which a value meets 4 others of its piece, 6 times the other lanes and a sum for every 256 values of the row (rows of more than 16384: 4 values for every
    4096, then 16 sums, which is fewer), and the square itself, at most 4 for every 1024 and 11, halved by the root; the mean's division, eps, root, reciprocal, p, two products, one more in hand: 8."""
    want_x = x + d.float() if d is not None else x
    assert torch.equal(got_x, want_x)
    n, cols = want_x.double() * gain.double(), x.shape[1]
    want, _ = exact_codes(n)
    assert (codes_of(q) - want).abs().max() <= 0.5 + 127 * 4.02 * U
    top = n.abs().amax(1)
    r = 1.0 / torch.sqrt((want_x.double() ** 2).mean(1) + eps)
    scale = torch.where(top >= TINY, top * r / 127.0, torch.zeros(()))
    chain = 4 * -(-cols // 1024) + 11
    assert ((q.scales.cpu().double() - scale).abs() <= scale * (chain / 2 + 8) * U).all()
    check_padding(q)


@pytest.mark.parametrize("add,gain_type", list(itertools.product([None, F32, BF16, F16], TYPES)))
@pytest.mark.parametrize("cols", [1, 5, 64, 255, 256, 1003, 1024, 2560, 4096, 5000, 9001, 20003])
def test_norm(cols, add, gain_type):
    g = gen(cols)
    x = torch.randn(7, cols, generator=g) * torch.exp(torch.randn(7, 1, generator=g))
    x[:, cols // 3] *= 20
    d = None if add is None else (0.3 * torch.randn(7, cols, generator=g)).to(add)
    gain = (1 + 0.1 * torch.randn(cols, generator=g)).to(gain_type)
    X, q = x.cuda(), B.Q8(7, cols)
    q.codes.fill_(55)
    B.op_rmsnorm_q8(X, gain.cuda(), 1e-6, q, add=None if d is None else d.cuda())
    check_norm(x, d, gain, 1e-6, q, X.cpu())


@pytest.mark.parametrize("cols", [64, 1003, 4096, 20003])
def test_norm_extremes(cols):
    """Rows with infinities and NaN in the stream, the addition or by their gain, sums of squares beyond fp32, rows of zeros and of tiny values; the others do not notice."""
    g = gen(5)
    x, d = torch.randn(12, cols, generator=g), torch.randn(12, cols, generator=g)
    x[1, cols - 1], d[2, 3], x[3, 0] = float("inf"), float("nan"), -float("inf")
    x[4], d[4] = 3e19, 0.0
    x[5], d[5] = 0.0, 0.0
    x[6], d[6] = 2.0 ** -121, 0.0
    x[7], d[7] = 1e-15, 0.0
    x[8], d[8] = 1.0, -1.0
    d[9, 5] = 1e10
    gain = 1 + 0.1 * torch.randn(cols, generator=g)
    X, q = x.cuda(), B.Q8(12, cols)
    B.op_rmsnorm_q8(X, gain.cuda(), 1e-6, q, add=d.cuda())
    bad = torch.zeros(12, dtype=torch.bool)
    bad[[1, 2, 3, 4]] = True
    assert torch.equal(torch.isnan(q.scales.cpu()), bad) and not codes_of(q)[bad].any()
    ok = B.Q8.of(q.codes[:, :cols][~bad.cuda()].contiguous(), q.scales[~bad.cuda()].contiguous())
    check_norm(x[~bad], d[~bad], gain, 1e-6, ok, X.cpu()[~bad])


@pytest.mark.parametrize("cols", [64, 1003, 4096, 20003])
def test_norm_of_rows_whose_normed_values_leave_fp32(cols):
    """A row whose stream and products with the gain are finite, but not its norm, is one with an infinity, as one is whose products with the gain are not; large rows
    whose norm is finite keep their codes."""
    x, gain = torch.zeros(4, cols), torch.ones(cols)
    gain[1], gain[2] = 3e38, 1e38 / cols ** 0.5
    x[0, 1] = 1.0                                               # normed: 3e38 sqrt(cols)
    x[1, 2], x[1, 3] = 1.7, 1e-3                                # about 1e38
    x[2, 1], x[2, 3] = 2.0, 1.0                                 # 6e38 before the division
    x[3] = 1.0
    x[3, 1] = 0.0
    q = B.Q8(4, cols)
    q.codes.fill_(55)
    X = x.cuda()
    B.op_rmsnorm_q8(X, gain.cuda(), 1e-6, q)
    assert torch.equal(X.cpu(), x)
    s, c = q.scales.cpu(), codes_of(q)
    assert torch.isnan(s[[0, 2]]).all() and not c[[0, 2]].any(), (s, c[:, :4])
    assert torch.isfinite(s[[1, 3]]).all() and c[1, 2] == 127 and c[3, 2] == 127
    ok = B.Q8.of(q.codes[1::2, :cols].contiguous(), q.scales[1::2].contiguous())
    check_norm(x[1::2], None, gain, 1e-6, ok, X.cpu()[1::2])


@pytest.mark.parametrize("eps", [1.5e-30, 1e-6, 0.9e30])
@pytest.mark.parametrize("cols", [64, 1003, 20003])
def test_norm_of_tiny_rows_at_both_ends_of_eps(cols, eps):
    """The limit of 2^-119 is on |x gain|, whatever eps makes of it: rows below it are zeros though their normed values may be far above, rows from it on keep their codes though
    their scale may be below fp32's normal numbers or 0.  The scale: as in check_norm, its last product and division off by half of the least subnormal more."""
    g = gen(cols)
    x = torch.zeros(7, cols)
    x[0], x[1], x[2] = TINY / 2, TINY, TINY
    x[1, 0], x[2, cols - 1] = 0.75 * TINY, -TINY
    x[3] = 1e-30 * torch.randn(cols, generator=g)
    x[4] = 1e-15 * torch.randn(cols, generator=g)
    x[5] = torch.randn(cols, generator=g)
    x[6, cols // 2] = TINY                                      # halved by the gain
    gain = torch.ones(cols)
    gain[cols // 2] = 0.5
    q = B.Q8(7, cols)
    q.codes.fill_(55)
    X = x.cuda()
    B.op_rmsnorm_q8(X, gain.cuda(), eps, q)
    n, e32 = x.double() * gain.double(), float(torch.tensor(eps, dtype=F32))
    want, _ = exact_codes(n)
    top = n.abs().amax(1)
    zeros = top < TINY
    assert zeros.tolist() == [True, False, False, False, False, False, True]
    assert not codes_of(q)[zeros].any() and not q.scales.cpu()[zeros].any()
    assert (codes_of(q) - want).abs().max() <= 0.5 + 127 * 4.02 * U
    scale = torch.where(zeros, torch.zeros(()).double(), top / torch.sqrt((x.double() ** 2).mean(1) + e32) / 127.0)
    chain = 4 * -(-cols // 1024) + 11
    assert ((q.scales.cpu().double() - scale).abs() <= scale * (chain / 2 + 8) * U + 1.01 * 2.0 ** -150).all()
    check_padding(q)


@pytest.mark.parametrize("cols", [5, 1003, 20003])
@pytest.mark.parametrize("gain_type", TYPES)
def test_norm_of_rows_whose_products_with_the_gain_leave_fp32(cols, gain_type):
    """1e17 times a gain of 3e38 is no number of fp32, though its norm may be one: a row with an infinity (half's gains are smaller).  The rows beside it do not notice."""
    top = 65504.0 if gain_type is F16 else 3e38
    gain = torch.ones(cols).to(gain_type)
    gain[1] = top
    x = torch.ones(3, cols)
    x[1] = 0.0
    x[1, 1], x[1, 2] = 1e17, 1e18                               # squares 1e36
    q = B.Q8(3, cols)
    B.op_rmsnorm_q8(x.cuda(), gain.cuda(), 1e-6, q)
    bad = torch.tensor([False, gain_type is not F16, False])
    assert torch.equal(torch.isnan(q.scales.cpu()), bad) and not codes_of(q)[bad].any()
    ok = B.Q8.of(q.codes[:, :cols][~bad.cuda()].contiguous(), q.scales[~bad.cuda()].contiguous())
    check_norm(x[~bad], None, gain, 1e-6, ok, x[~bad])


@pytest.mark.parametrize("cols", [64, 500, 1003, 2048, 4096, 9000, 12288, 16384, 20003])
def test_rows_do_not_depend_on_the_rows_beside_them(cols):
    """One row, a hundred and two thousand take different numbers of threads a row: same bits of stream, codes and scales."""
    x, d, gain = torch.randn(2000, cols, device="cuda"), torch.randn(2000, cols, device="cuda").to(BF16), torch.randn(cols, device="cuda")
    X, q, p = x.clone(), B.Q8(2000, cols), B.Q8(2000, cols)
    B.op_rmsnorm_q8(X, gain, 1e-6, q, add=d)
    B.op_quantize_q8(d, p)
    for n in (1, 100):
        Y, r = x[:n].clone(), B.Q8(n, cols)
        B.op_rmsnorm_q8(Y, gain, 1e-6, r, add=d[:n])
        assert torch.equal(Y, X[:n]) and torch.equal(r.codes, q.codes[:n]) and torch.equal(r.scales, q.scales[:n])
        B.op_quantize_q8(d[:n], r)
        assert torch.equal(r.codes, p.codes[:n]) and torch.equal(r.scales, p.scales[:n])


def test_norm_strides():
    """Stream, addition and codes as views of larger buffers: nothing beside the rows is written, the additions of other rows are not read."""
    g = gen(6)
    for cols in (5, 130, 1003, 5001):
        buf, add = torch.randn(9, cols + 7, generator=g).cuda(), torch.randn(9, cols + 3, generator=g).to(BF16).cuda()
        before, gain = buf.clone(), torch.ones(cols, device="cuda", dtype=F16)
        x = buf[2:7, 3:3 + cols].cpu()
        q = B.Q8(9, cols).first(5)
        B.op_rmsnorm_q8(buf[2:7, 3:3 + cols], gain, 1e-5, q, add=add[1:6, 1:1 + cols])
        check_norm(x, add[1:6, 1:1 + cols].cpu(), gain.cpu(), 1e-5, q, buf[2:7, 3:3 + cols].cpu())
        buf[2:7, 3:3 + cols] = before[2:7, 3:3 + cols]
        assert torch.equal(buf, before)


# ------------------------------------------------------------------------------------------------------------------ products

def operands(M, N, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda n: torch.randint(-128, 128, (n, K), generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    a, w = rnd(M), rnd(N)
    sa = torch.rand(M, generator=g, device="cuda") * 1e-2 + 1e-4
    sw = (torch.rand(N, generator=g, device="cuda") + 0.1) / (K ** 0.5 * 40)
    return a, sa, w, sw


def product(a, sa, w, sw):
    """In 64 bits, by panels: integer sums below 2^31 are exact."""
    wt = w.double().t().contiguous()
    return torch.cat([(a[i:i + 2048].double() @ wt) * sa[i:i + 2048].double()[:, None] * sw.double() for i in range(0, len(a), 2048)])


EPILOGUES = [(B.EPI_STORE, BF16), (B.EPI_STORE, F16), (B.EPI_STORE_F32, F32), (B.EPI_RESIDUAL, F32), (B.EPI_SWIGLU, BF16), (B.EPI_SWIGLU, F16)]


def check_product(epilogue, dtype, out, old, y):
    """fp32: the sum's conversion and two products, 3 u; the residual's addition one of the result.  SwiGLU: gate and up 3 u each, 1 + e and two products 3 u, the reciprocal and the
    exponential an ulp (2 u) each, and the exponent g log2(e): gate's 3 u, its own product's and constant's 1.5 u, in all 4.5 u |g|.  Where 1 + e leaves the reciprocal's range
    (2^126, |g| > 87.3) the result is 0 for what is below 88 2^-126 |up| < 1.1e-36 |up|.  16 bits: half a step more, and half the least subnormal."""
    if epilogue == B.EPI_SWIGLU:
        f = y.shape[1] // 2
        gate, up = y[:, :f], y[:, f:]
        want = gate * torch.sigmoid(gate) * up
        err = want.abs() * (13.1 + 4.6 * gate.abs()) * U + 1.1e-36 * up.abs()
    elif epilogue == B.EPI_RESIDUAL:
        want = old.double() + y
        err = y.abs() * 3.01 * U + want.abs() * U
    else:
        want, err = y, y.abs() * 3.01 * U
    if dtype is F16:
        want = want.clamp(-65504, 65504)
    err = err + (want.abs() + err) * half_step(dtype) + smallest(dtype)
    off = (out.double() - want).abs() - err
    assert torch.isfinite(out).all() and off.max() <= 0, (float(off.max()), int((off > 0).sum()))


def run_product(M, N, K, epilogue, dtype, seed=0):
    a, sa, w, sw = operands(M, N, K, seed)
    cols = N // 2 if epilogue == B.EPI_SWIGLU else N
    old = torch.randn(M, cols, device="cuda") if epilogue == B.EPI_RESIDUAL else torch.empty(M, cols, dtype=dtype, device="cuda")
    out = old.clone()
    B.op_gemm_q8(epilogue, B.Q8.of(a, sa), B.Q8.of(w, sw), out)
    check_product(epilogue, dtype, out, old, product(a, sa, w, sw))


SIZES = [(1, 2, 1), (1, 64, 64), (1, 4096, 256), (2, 66, 129), (3, 1000, 500), (7, 130, 1003), (17, 48, 128), (24, 514, 4096), (33, 2560, 640), (64, 62, 12288), (65, 4096, 384),
         (100, 1026, 257), (129, 6144, 1024), (200, 2000, 2047), (391, 4096, 1024), (513, 258, 320), (777, 2562, 1003), (1154, 2560, 512), (2000, 130, 96),
         (3000, 1024, 640), (4100, 6144, 640), (5000, 1234, 333),
         (18, 17076, 785), (130, 5648, 2565), (19713, 70, 1426), (517, 20866, 141), (133, 22094, 1797), (17800, 698, 130), (1208, 10764, 266),
         (17185, 648, 390), (33, 8630, 68), (517, 20142, 66)]         # tests/test_q8_plan.py: every tile


@pytest.mark.parametrize("epilogue,dtype", EPILOGUES)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_gemm(M, N, K, epilogue, dtype):
    run_product(M, N, K, epilogue, dtype)


ODD_SIZES = [(5, 31, 40), (300, 257, 70), (1543, 2501, 1003), (2600, 1281, 130)]


@pytest.mark.parametrize("epilogue,dtype", EPILOGUES)
def test_gemm_odd_widths(epilogue, dtype):
    """Outputs whose rows begin at no multiple of anything, and last tiles of a single column."""
    for M, N, K in ODD_SIZES:
        if epilogue == B.EPI_SWIGLU:
            N *= 2
        run_product(M, N, K, epilogue, dtype)


@pytest.mark.parametrize("epilogue,dtype", EPILOGUES)
def test_gemm_that_begins_anywhere_in_k(epilogue, dtype):
    """Up to 512 rows by weights whose rows are a multiple of 4 KiB apart: column tiles begin at different slices of K and come round."""
    for M, N, K in ((70, 1026, 4096), (300, 2048, 4000), (512, 514, 8192), (200, 260, 12288), (40, 24576, 4096)):
        run_product(M, N, K, epilogue, dtype)


# rows, columns, K: tests/test_q8_plan.py: every tile, with weights' rows a multiple of 4 KiB apart
TURN_SIZES = [(460, 21890, 4000), (386, 22126, 4096), (502, 16502, 4000), (390, 16564, 4000), (391, 8526, 4000), (475, 8758, 4000), (455, 8222, 4000), (400, 8228, 4000),
              (457, 4140, 4000), (455, 2078, 4000), (481, 1028, 4000), (10, 16764, 4000), (482, 524, 3981), (70, 130, 4000), (341, 3940, 2332), (87, 16420, 2478),
              (108, 14410, 1929), (512, 24576, 4096), (391, 24576, 4096), (450, 4096, 12288)]


@pytest.mark.parametrize("epilogue,dtype", EPILOGUES)
@pytest.mark.parametrize("M,N,K", TURN_SIZES)
def test_gemm_that_begins_anywhere_in_k_on_every_tile(M, N, K, epilogue, dtype):
    """The same on all tiles; rows that are shorter than a multiple of 4 KiB have gaps behind them, whose bytes do not count.  The same bits as with rows that are 128 codes further
    apart, where every tile begins at K's start."""
    a, sa, w, sw = operands(M, N, K, 7)
    width, apart = (K + 127) // 128 * 128, (K + 4095) // 4096 * 4096

    def spread(stride):
        store = torch.full((N, stride), 99, dtype=torch.int8, device="cuda")
        store[:, :K], store[:, K:width] = w, 0
        q = B.Q8(0, K)
        q._set(store, sw, K)
        return q
    cols = N // 2 if epilogue == B.EPI_SWIGLU else N
    old = torch.randn(M, cols, device="cuda").to(dtype)
    out, straight, A = old.clone(), old.clone(), B.Q8.of(a, sa)
    B.op_gemm_q8(epilogue, A, spread(apart), out)
    check_product(epilogue, dtype, out, old, product(a, sa, w, sw))
    B.op_gemm_q8(epilogue, A, spread(apart + 128), straight)
    assert torch.equal(out, straight)


@pytest.mark.parametrize("M", [1, 12, 100, 600])
def test_weights_of_nearly_four_gib(M):
    """Offsets within the weights pass 31 bits: columns in front of 2 GiB, around it and the last ones, on the kernel of few rows and on small and large tiles."""
    N, K = 1000000, 4096
    W = B.Q8(N, K)
    g = torch.Generator(device="cuda").manual_seed(M)
    for i in range(0, N, 100000):
        W.codes[i:i + 100000].random_(-128, 128, generator=g)
    W.scales.uniform_(1e-5, 1e-4, generator=g)
    a, sa, _, _ = operands(M, 1, K, 8)
    A = B.Q8.of(a, sa)
    old = torch.randn(M, N, device="cuda")
    out = old.clone()
    B.op_gemm_q8(B.EPI_RESIDUAL, A, W, out)
    for at in (0, (1 << 31) // K - 150, N - 300):
        c = slice(at, at + 300)
        check_product(B.EPI_RESIDUAL, F32, out[:, c], old[:, c], product(a, sa, W.codes[c], W.scales[c]))
    del out, old
    h = torch.empty(M, N // 2, dtype=BF16, device="cuda")
    B.op_gemm_q8(B.EPI_SWIGLU, A, W, h)
    for at in (0, (1 << 30) // K, (1 << 31) // K - N // 2, N // 2 - 300):
        rows = torch.cat([torch.arange(at, at + 300), torch.arange(N // 2 + at, N // 2 + at + 300)]).cuda()
        check_product(B.EPI_SWIGLU, BF16, h[:, at:at + 300], None, product(a, sa, W.codes[rows], W.scales[rows]))


@pytest.mark.parametrize("M", [1, 8, 9, 16, 17, 32, 33, 64, 65])
def test_gemm_around_the_kernel_of_few_rows(M):
    for N, K in ((64, 70), (4096, 1024), (4098, 1024), (8192, 1024), (8194, 1000), (2046, 2176), (2048, 2176), (512, 4224)):
        run_product(M, N, K, B.EPI_RESIDUAL, F32)
        run_product(M, N, K, B.EPI_SWIGLU, F16)


@pytest.mark.parametrize("M,N", [(1, 64), (130, 300)])
def test_gemm_largest_sums(M, N):
    """The longest rows of the largest codes: 2^14 * 131071 just fits 32 bits, in both signs."""
    K = 131071
    a, w = torch.full((M, K), -128, dtype=torch.int8, device="cuda"), torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    w[N // 2:] = 127
    one = lambda n: torch.full((n,), 0.5, device="cuda")  # noqa: E731
    out = torch.empty(M, N, device="cuda")
    B.op_gemm_q8(B.EPI_STORE_F32, B.Q8.of(a, one(M)), B.Q8.of(w, one(N)), out)
    want = torch.where(torch.arange(N) < N // 2, 16384.0 * K / 4, -16256.0 * K / 4).to(F32)
    assert torch.equal(out.cpu(), want.expand(M, N))


@pytest.mark.parametrize("epilogue,dtype", EPILOGUES)
def test_gemm_strides_and_neighbours(epilogue, dtype):
    """Operands as row ranges of larger buffers whose rows have gaps, an output within a larger one: nothing beside it is written, what stands between the operands' rows is not read
    into the result."""
    for M, N, K in ((3, 70, 130), (150, 322, 500), (700, 1026, 256)):
        a, sa, w, sw = operands(M, N, K, 3)
        width = (K + 127) // 128 * 128

        def spread(codes, scales):
            store = torch.full((len(codes) + 2, width + 48), 99, dtype=torch.int8, device="cuda")
            store[1:-1, :K], store[1:-1, K:width] = codes, 0
            q = B.Q8(0, K)
            q._set(store[1:-1], scales.clone(), K)
            return q
        cols = N // 2 if epilogue == B.EPI_SWIGLU else N
        buf = torch.randn(M + 2, cols + 11, device="cuda").to(dtype)
        before = buf.clone()
        B.op_gemm_q8(epilogue, spread(a, sa), spread(w, sw), buf[1:-1, 5:5 + cols])
        check_product(epilogue, dtype, buf[1:-1, 5:5 + cols], before[1:-1, 5:5 + cols], product(a, sa, w, sw))
        buf[1:-1, 5:5 + cols] = before[1:-1, 5:5 + cols]
        assert torch.equal(buf, before)


@pytest.mark.parametrize("epilogue,dtype", EPILOGUES)
def test_gemm_rows_without_a_scale(epilogue, dtype):
    """A row of A, or of W, whose scale is NaN makes its row, or column, NaN, and no other; half keeps the NaN and saturates otherwise."""
    for M, N, K in ((5, 66, 100), (300, 514, 300)):
        a, sa, w, sw = operands(M, N, K, 4)
        a[2], w[7] = 0, 0
        sa[2], sw[7] = float("nan"), float("nan")
        sa[3] = 1e6
        cols = N // 2 if epilogue == B.EPI_SWIGLU else N
        old = torch.zeros(M, cols, dtype=dtype, device="cuda")
        out = old.clone()
        B.op_gemm_q8(epilogue, B.Q8.of(a, sa), B.Q8.of(w, sw), out)
        bad = torch.zeros(M, cols, dtype=torch.bool, device="cuda")
        bad[2], bad[:, 7] = True, True
        assert torch.equal(torch.isnan(out), bad)
        if dtype is F16:
            assert out[3][~bad[3]].abs().max() == 65504
        sa[2], sw[7], sa[3] = 0.0, 0.0, 1e-3                     # nothing else differs
        clean = old.clone()
        B.op_gemm_q8(epilogue, B.Q8.of(a, sa), B.Q8.of(w, sw), clean)
        rest = ~bad
        rest[3] = False
        assert torch.equal(out[rest], clean[rest])


def test_gemm_is_the_same_at_every_size_of_the_batch():
    """Sums are exact, so a row's bits do not depend on the rows beside it, whatever tiles they take."""
    a, sa, w, sw = operands(3000, 1030, 777, 5)
    W = B.Q8.of(w, sw)
    for epilogue, dtype in EPILOGUES:
        cols = 515 if epilogue == B.EPI_SWIGLU else 1030
        A = B.Q8.of(a, sa)
        full = torch.zeros(3000, cols, dtype=dtype, device="cuda")
        B.op_gemm_q8(epilogue, A, W, full)
        for m in (1, 2, 16, 40, 100, 300, 1000):
            part = torch.zeros(m + 1, cols, dtype=dtype, device="cuda")
            part[m] = 3.0
            B.op_gemm_q8(epilogue, A.first(m), W, part[:m])
            assert torch.equal(part[:m], full[:m]) and (part[m] == 3).all(), (epilogue, m)


@pytest.mark.parametrize("epilogue,dtype", EPILOGUES)
@pytest.mark.parametrize("N,K", [(1030, 777), (512, 4224), (9000, 700), (6000, 1000), (4096, 1024)])
def test_gemm_of_a_stream_is_the_same_at_every_size_of_the_batch(N, K, epilogue, dtype):
    """The same over an output that holds numbers: what is added to the stream is rounded before the addition in the kernel of few rows and in all tiles.  The
    first takes up to 8, 16, 32 or 64 rows here."""
    a, sa, w, sw = operands(2100, N, K, 6)
    A, W, cols = B.Q8.of(a, sa), B.Q8.of(w, sw), N // 2 if epilogue == B.EPI_SWIGLU else N
    old = torch.randn(2100, cols, generator=torch.Generator(device="cuda").manual_seed(N), device="cuda").to(dtype)
    full = old.clone()
    B.op_gemm_q8(epilogue, A, W, full)
    for m in (1, 8, 9, 16, 17, 32, 33, 64, 65, 200, 500, 1100):
        part = old[:m + 1].clone()
        B.op_gemm_q8(epilogue, A.first(m), W, part[:m])
        assert torch.equal(part[:m], full[:m]) and torch.equal(part[m], old[m]), (m, int((part[:m] != full[:m]).sum()))


@pytest.mark.parametrize("epilogue,dtype", EPILOGUES)
def test_gemm_of_one_column(epilogue, dtype):
    for M, N, K in ((1, 1, 3), (8, 3, 1), (65, 1, 130), (300, 5, 1003), (5000, 1, 128), (1, 1, 131071)):
        run_product(M, N * (2 if epilogue == B.EPI_SWIGLU else 1), K, epilogue, dtype)


def test_rows_behind_four_gib():
    """Rows whose offsets pass 32 bits, in values and in bytes: the last ones give what they give by themselves."""
    rows, cols, tail = 530000, 8192, 1000
    x = torch.empty(rows, cols, dtype=BF16, device="cuda")
    x.view(torch.int16).random_(0x3c00, 0x3f80)                # numbers from 2^-7 up to 1
    q, part = B.Q8(rows, cols), B.Q8(tail, cols)
    B.op_quantize_q8(x, q)
    B.op_quantize_q8(x[-tail:], part)
    assert torch.equal(q.codes[-tail:], part.codes) and torch.equal(q.scales[-tail:], part.scales)
    _, _, w, sw = operands(1, 66, cols, 10)
    W = B.Q8.of(w, sw)
    out, alone = torch.empty(rows, 66, device="cuda"), torch.empty(tail, 66, device="cuda")
    B.op_gemm_q8(B.EPI_STORE_F32, q, W, out)
    B.op_gemm_q8(B.EPI_STORE_F32, part, W, alone)
    assert torch.equal(out[-tail:], alone)
    check_product(B.EPI_STORE_F32, F32, alone, None, product(part.codes, part.scales, w, sw))
    back = torch.empty(rows, cols, dtype=F16, device="cuda")
    B.op_dequantize_q8(q, back)
    assert torch.equal(back[-tail:].double(), (part.codes.float() * part.scales[:, None]).half().double())
    del x, back
    X = torch.ones(rows, cols, device="cuda")
    X[-tail:] = torch.randn(tail, cols, generator=gen(11)).cuda()
    last = X[-tail:].clone()
    gain = torch.ones(cols, device="cuda")
    B.op_rmsnorm_q8(X, gain, 1e-6, q, add=torch.full((rows, cols), 0.5, dtype=F16, device="cuda"))
    B.op_rmsnorm_q8(last, gain, 1e-6, part, add=torch.full_like(last, 0.5))
    assert torch.equal(X[-tail:], last) and torch.equal(q.codes[-tail:], part.codes) and torch.equal(q.scales[-tail:], part.scales)


def test_empty_calls():
    q, w = B.Q8(0, 256), B.Q8(300, 256)
    B.op_quantize_q8(torch.empty(0, 256, device="cuda"), q)
    B.op_rmsnorm_q8(torch.empty(0, 256, device="cuda"), torch.ones(256, device="cuda"), 1e-6, q)
    B.op_dequantize_q8(q, torch.empty(0, 256, device="cuda"))
    w.codes.zero_()
    w.scales.zero_()
    B.op_gemm_q8(B.EPI_STORE_F32, q, w, torch.empty(0, 300, device="cuda"))
    B.op_gemm_q8(B.EPI_STORE_F32, w, q, torch.empty(300, 0, device="cuda"))
    torch.cuda.synchronize()


def test_binding_refusals():
    q, w = B.Q8(4, 256), B.Q8(6, 256)
    x = torch.zeros(4, 256, device="cuda")
    bad = [lambda: B.op_quantize_q8(x[:3], q), lambda: B.op_quantize_q8(x[:, :255], q), lambda: B.op_quantize_q8(x.double(), q), lambda: B.op_quantize_q8(x.t(), q),
           lambda: B.op_quantize_q8(x.cpu(), q), lambda: B.op_dequantize_q8(q, x[:, ::2]), lambda: B.op_dequantize_q8(q, x.int()),
           lambda: B.op_rmsnorm_q8(x.half(), x[0], 1e-6, q), lambda: B.op_rmsnorm_q8(x, x[0, :255], 1e-6, q), lambda: B.op_rmsnorm_q8(x, x[0].cpu(), 1e-6, q),
           lambda: B.op_rmsnorm_q8(x, x[0], 0.0, q), lambda: B.op_rmsnorm_q8(x, x[0], 1e-6, q, add=x[:2]),
           lambda: B.op_gemm_q8(B.EPI_STORE, q, w, torch.zeros(4, 6, device="cuda")), lambda: B.op_gemm_q8(B.EPI_STORE_F32, q, w, torch.zeros(4, 5, device="cuda")),
           lambda: B.op_gemm_q8(B.EPI_RESIDUAL, q, w, torch.zeros(6, 4, device="cuda").t()), lambda: B.op_gemm_q8(7, q, w, torch.zeros(4, 6, device="cuda")),
           lambda: B.op_gemm_q8(B.EPI_STORE_F32, q, B.Q8(6, 255), torch.zeros(4, 6, device="cuda")), lambda: B.Q8(3, 0), lambda: q.first(5), lambda: q.first(-1),
           lambda: B.Q8.of(x, x[:, 0]), lambda: B.Q8.of(q.codes, x[0, :3])]
    for f in bad:
        with pytest.raises(B.PrismError):
            f()


# ------------------------------------------------------------------------------------------------------------------ together

def block(X, D, gain, W1, W2, q, h, h8, out):
    """A feed-forward block: what a layer calls."""
    B.op_rmsnorm_q8(X, gain, 1e-6, q, add=D)
    B.op_gemm_q8(B.EPI_SWIGLU, q, W1, h)
    B.op_quantize_q8(h, h8)
    B.op_gemm_q8(B.EPI_RESIDUAL, h8, W2, out)


def block_buffers(rows, hidden, ffn, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    W1, W2 = B.Q8(2 * ffn, hidden), B.Q8(hidden, ffn)
    B.op_quantize_q8((rnd(2 * ffn, hidden) * 0.1).to(BF16), W1)
    B.op_quantize_q8((rnd(hidden, ffn) * 0.1).to(BF16), W2)
    X, D, gain = rnd(rows, hidden), rnd(rows, hidden).to(dtype), (1 + 0.1 * rnd(hidden)).to(BF16)
    return X, D, gain, W1, W2, B.Q8(rows, hidden), torch.empty(rows, ffn, dtype=dtype, device="cuda"), B.Q8(rows, ffn), X.clone()


@pytest.mark.parametrize("rows,hidden,ffn,dtype", [(1, 256, 640, BF16), (37, 500, 1003, F16), (700, 1024, 2816, BF16)])
def test_a_block(rows, hidden, ffn, dtype):
    """Each step against its own definition on what the step before it left."""
    buf = block_buffers(rows, hidden, ffn, dtype, 7)
    X, D, gain, W1, W2, q, h, h8, out = buf
    x, old = X.cpu(), out.clone()
    block(*buf)
    check_norm(x, D.cpu(), gain.cpu(), 1e-6, q, X.cpu())
    c = lambda r: r.codes[:, :r.cols]  # noqa: E731
    check_product(B.EPI_SWIGLU, dtype, h, None, product(c(q), q.scales, c(W1), W1.scales))
    want, _ = exact_codes(host(h))
    assert torch.equal(codes_of(h8), torch.round(want))
    check_product(B.EPI_RESIDUAL, F32, out, old, product(c(h8), h8.scales, c(W2), W2.scales))


def test_a_block_captured_and_replayed():
    """One graph, replayed on changing inputs between eager work: every replay gives the eager calls' bits.  Two graphs of the same weights on two streams do not meet."""
    eager, a, b = (block_buffers(130, 512, 1408, F16, 8) for _ in range(3))
    for buf in (eager, a, b):
        block(*buf)
    torch.cuda.synchronize()
    graphs = []
    for buf in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            block(*buf)
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for turn in range(4):
        x, d = torch.randn(130, 512, device="cuda") * (turn + 1), torch.randn(130, 512, device="cuda").half()
        for buf in (eager, a, b):
            buf[0].copy_(x)
            buf[1].copy_(d)
            buf[8].copy_(x)
        block(*eager)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for buf in (a, b):
            assert torch.equal(buf[8], eager[8]) and torch.equal(buf[0], eager[0]) and torch.equal(buf[7].codes, eager[7].codes), turn


def test_blocks_in_two_threads():
    """Two threads, a stream each, the same weights: nothing is shared but what is read."""
    import threading
    want = [block_buffers(60 + 300 * i, 512, 1408, F16, 12 + i) for i in range(2)]
    got = [block_buffers(60 + 300 * i, 512, 1408, F16, 12 + i) for i in range(2)]
    shared = got[0][3:5]
    torch.cuda.synchronize()

    def run(i):
        buf = got[i][:3] + shared + got[i][5:]
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                block(*buf)
            torch.cuda.current_stream().synchronize()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for i in range(2):
        buf = want[i][:3] + shared + want[i][5:]
        for _ in range(20):
            block(*buf)
        assert torch.equal(got[i][0], want[i][0]) and torch.equal(got[i][8], want[i][8]) and torch.equal(got[i][7].codes, want[i][7].codes)


def test_weights_in_eight_bits_stand_for_the_weights():
    """What quantisation costs: every weight is within half a step of its code, so a product of rows that are codes already is off by at most the sum of |a| times half a step."""
    g = gen(9)
    w = torch.randn(300, 640, generator=g).to(BF16)
    W = B.Q8(300, 640)
    B.op_quantize_q8(w.cuda(), W)
    back = torch.empty(300, 640, device="cuda")
    B.op_dequantize_q8(W, back)
    scale = host(W.scales)[:, None]
    assert ((host(back) - w.double()).abs() <= scale * (0.5 + 127 * 3 * U)).all()
    a, sa, _, _ = operands(50, 2, 640, 9)
    out = torch.empty(50, 300, device="cuda")
    B.op_gemm_q8(B.EPI_STORE_F32, B.Q8.of(a, sa), W, out)
    ad = host(a) * host(sa)[:, None]
    limit = ad.abs().sum(1, keepdim=True) * scale.t() * (0.5 + 127 * 7 * U)
    assert ((host(out) - ad @ w.double().t()).abs() <= limit).all()
