"""Operators of a layer whose products run in 8-bit integers, as cases with stated inputs, plain forms and exact results.

Four kinds of work: `norm` (residual addition, RMSNorm, rows of 8-bit codes with a scale each), `quant` (rows to codes and scales),
`gemm` (product of two matrices of codes, with the scales and an epilogue) and `ffn` (a feed-forward block of all of them in a row).

A row x of codes stands for code * scale with scale = max|x| / 127 and code = x / scale rounded to the nearest integer, ties to even.
Codes are returned as the values they stand for, in bf16.
"""
import math

import torch

own = False

TORCH = {"f16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


def listed():
    return [
        # the norm of a serving step: 24 sequences, a token each, 8B hidden size, the attention block's output still to be added: latency
        {"name": "norm_step", "kind": "norm", "rows": 24, "cols": 4096, "add": "bf16", "gain": "bf16"},
        # the norm of a pruned pool of documents, 8B hidden size: bandwidth
        {"name": "norm_pool", "kind": "norm", "rows": 11584, "cols": 4096, "add": "f16", "gain": "bf16"},
        # rows of an odd length, everything in fp32
        {"name": "norm_odd", "kind": "norm", "rows": 4099, "cols": 1003, "add": "fp32", "gain": "fp32"},
        # the SwiGLU output of a few last tokens, 8B shape: latency
        {"name": "quant_step", "kind": "quant", "rows": 7, "cols": 12288, "dtype": "f16"},
        # the SwiGLU output of a pool, 8B shape: bandwidth
        {"name": "quant_pool", "kind": "quant", "rows": 11584, "cols": 12288, "dtype": "bf16"},
        # the O projection of one token, 8B shape: the smallest product, its weights' bytes
        {"name": "gemm_token", "kind": "gemm", "epilogue": "residual", "rows": 1, "n": 4096, "k": 4096, "dtype": "fp32"},
        # gate and up of a serving step of 24 tokens, 8B shape: bandwidth
        {"name": "gemm_step", "kind": "gemm", "epilogue": "swiglu", "rows": 24, "n": 24576, "k": 4096, "dtype": "bf16"},
        # the down projection of a pool's last tokens, 8B shape
        {"name": "gemm_last", "kind": "gemm", "epilogue": "residual", "rows": 100, "n": 4096, "k": 12288, "dtype": "fp32"},
        # the q/k/v projection of a few short passages, 0.6B shape, fp32 for the head norms and the rotation behind it
        {"name": "gemm_qkv", "kind": "gemm", "epilogue": "store_f32", "rows": 391, "n": 4096, "k": 1024, "dtype": "fp32"},
        # odd sizes in all three directions
        {"name": "gemm_odd", "kind": "gemm", "epilogue": "store", "rows": 1543, "n": 2501, "k": 1003, "dtype": "f16"},
        # gate and up of a pruned pool, 8B shape: matrix work
        {"name": "gemm_pool", "kind": "gemm", "epilogue": "swiglu", "rows": 11584, "n": 24576, "k": 4096, "dtype": "f16"},
        # a whole feed-forward block, 4B shape, from the stream to what the next norm adds to it
        {"name": "ffn_pool", "kind": "ffn", "rows": 3699, "cols": 2560, "ffn": 9728, "dtype": "bf16", "gain": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "quant", "gemm", "gemm", "gemm", "ffn"])
    width = lambda lo, hi: rng.choice([lambda v: v, lambda v: -(-v // 8) * 8, lambda v: -(-v // 128) * 128])(_log_int(rng, lo, hi))  # noqa: E731
    if kind in ("norm", "quant"):
        cols = width(64, 12288)
        case = {"kind": kind, "rows": _log_int(rng, 1, min(100000, 100000000 // cols)), "cols": cols}
        if kind == "quant":
            return {**case, "dtype": rng.choice(["f16", "bf16", "fp32"])}
        return {**case, "add": rng.choice(["", "f16", "bf16", "fp32"]), "gain": rng.choice(["f16", "bf16", "fp32"])}
    if kind == "ffn":
        cols, ffn = width(128, 4096), width(256, 12288)
        return {"kind": kind, "rows": _log_int(rng, 1, min(20000, 360000000000 // (cols * ffn))), "cols": cols, "ffn": ffn,
                "dtype": rng.choice(["f16", "bf16"]), "gain": rng.choice(["f16", "bf16", "fp32"])}
    epilogue = rng.choice(["store", "store_f32", "residual", "swiglu"])
    n, k = width(64, 24576), width(64, 12288)
    return {"kind": kind, "epilogue": epilogue, "rows": _log_int(rng, 1, min(20000, 1100000000000 // (n * k))), "n": n + n % 2 if epilogue == "swiglu" else n, "k": k,
            "dtype": rng.choice(["f16", "bf16"]) if epilogue in ("store", "swiglu") else "fp32"}


def _codes(x):
    """Rows of codes and their scales, from rows of numbers: how a state's codes come about."""
    scale = x.abs().amax(1).float() / 127.0
    return torch.round(x.float() / scale[:, None]).clamp_(-127, 127).to(torch.int8), scale


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)  # noqa: E731
    kind, s = case["kind"], {"case": case}

    def stream(rows, cols):
        """A residual stream: a few channels are much larger than the others, rows differ in size."""
        x = randn(rows, cols) * torch.exp(0.5 * randn(rows, 1))
        return torch.where(torch.rand(cols, generator=g, device="cuda") < 0.005, 20.0, 1.0) * x

    if kind in ("norm", "ffn"):
        s["x"] = stream(case["rows"], case["cols"])
        add = case.get("add", case.get("dtype"))
        s["d"] = (0.3 * randn(case["rows"], case["cols"])).to(TORCH[add]) if add else None
        s["gain"] = (1 + 0.1 * randn(case["cols"])).to(TORCH[case["gain"]])
    if kind == "quant":
        s["x"] = (randn(case["rows"], case["cols"]) * randn(case["rows"], case["cols"])).to(TORCH[case["dtype"]])
    if kind == "gemm":
        s["a"], s["sa"] = _codes(stream(case["rows"], case["k"]))
        s["w"], s["sw"] = _codes(0.02 * randn(case["n"], case["k"]))
        cols = case["n"] // 2 if case["epilogue"] == "swiglu" else case["n"]
        s["out"] = randn(case["rows"], cols) if case["epilogue"] == "residual" else torch.empty(case["rows"], cols, dtype=TORCH[case["dtype"]], device="cuda")
    if kind == "ffn":
        s["w1"], s["sw1"] = _codes(0.02 * randn(2 * case["ffn"], case["cols"]))
        s["w2"], s["sw2"] = _codes(0.02 * randn(case["cols"], case["ffn"]))
        s["out"] = torch.empty(case["rows"], case["cols"], dtype=TORCH[case["dtype"]], device="cuda")
    if own:
        # the handles that a program keeps: weights and activations in 8 bits, buffers for results
        from paper_2510_15620_amd import binding as B
        if kind in ("norm", "quant"):
            s["q"] = B.Q8(case["rows"], case["cols"])
            s["values"] = torch.empty(case["rows"], case["cols"], dtype=torch.bfloat16, device="cuda")
        if kind == "gemm":
            s["A"], s["W"] = B.Q8.of(s["a"], s["sa"]), B.Q8.of(s["w"], s["sw"])
        if kind == "ffn":
            s["q"], s["h8"] = B.Q8(case["rows"], case["cols"]), B.Q8(case["rows"], case["ffn"])
            s["h"] = torch.empty(case["rows"], case["ffn"], dtype=TORCH[case["dtype"]], device="cuda")
            s["W1"], s["W2"] = B.Q8.of(s["w1"], s["sw1"]), B.Q8.of(s["w2"], s["sw2"])
    return s


def _quantise(x):
    """Codes (as fp32 numbers) and scales of rows of fp32 values."""
    scale = x.abs().amax(1, keepdim=True) / 127.0
    return torch.round(x / scale).clamp(-127.0, 127.0), scale


def _norm(s):
    """The stream with the addition, and the normed rows in fp32."""
    if s["d"] is not None:
        s["x"] += s["d"].float()
    x = s["x"]
    return x / torch.sqrt((x * x).mean(1, keepdim=True) + EPS) * s["gain"].float()


def _product(codes, scale, w, sw):
    return torch.matmul(codes, w.float().t()) * scale * sw


def _swiglu(y):
    gate, up = y.chunk(2, 1)
    return gate / (1.0 + torch.exp(-gate)) * up


def _plain(s):
    c = s["case"]
    if c["kind"] == "norm":
        codes, scale = _quantise(_norm(s))
        return [s["x"], scale[:, 0], (codes * scale).to(torch.bfloat16)]
    if c["kind"] == "quant":
        codes, scale = _quantise(s["x"].float())
        return [scale[:, 0], (codes * scale).to(torch.bfloat16)]
    if c["kind"] == "ffn":
        codes, scale = _quantise(_norm(s))
        h = _swiglu(_product(codes, scale, s["w1"], s["sw1"])).to(TORCH[c["dtype"]])
        codes, scale = _quantise(h.float())
        s["out"][:] = _product(codes, scale, s["w2"], s["sw2"])
        return [s["x"], s["out"]]
    y = _product(s["a"].float(), s["sa"][:, None], s["w"], s["sw"])
    if c["epilogue"] == "residual":
        s["out"] += y
    else:
        s["out"][:] = _swiglu(y) if c["epilogue"] == "swiglu" else y
    return [s["out"]]


def run(s):
    if not own:
        return _plain(s)
    from paper_2510_15620_amd import binding as B
    c = s["case"]
    if c["kind"] == "norm":
        B.op_rmsnorm_q8(s["x"], s["gain"], EPS, s["q"], add=s["d"])
        B.op_dequantize_q8(s["q"], s["values"])
        return [s["x"], s["q"].scales, s["values"]]
    if c["kind"] == "quant":
        B.op_quantize_q8(s["x"], s["q"])
        B.op_dequantize_q8(s["q"], s["values"])
        return [s["q"].scales, s["values"]]
    if c["kind"] == "ffn":
        B.op_rmsnorm_q8(s["x"], s["gain"], EPS, s["q"], add=s["d"])
        B.op_gemm_q8(B.EPI_SWIGLU, s["q"], s["W1"], s["h"])
        B.op_quantize_q8(s["h"], s["h8"])
        B.op_gemm_q8(B.EPI_STORE, s["h8"], s["W2"], s["out"])
        return [s["x"], s["out"]]
    epilogue = {"store": B.EPI_STORE, "store_f32": B.EPI_STORE_F32, "residual": B.EPI_RESIDUAL, "swiglu": B.EPI_SWIGLU}[c["epilogue"]]
    B.op_gemm_q8(epilogue, s["A"], s["W"], s["out"])
    return [s["out"]]


def work(case):
    rows, size = case["rows"], {"": 0, "f16": 2, "bf16": 2, "fp32": 4}
    if case["kind"] == "quant":         # rows in; values and a scale a row out
        return {"bytes": rows * (case["cols"] * (size[case["dtype"]] + 2) + 4), "flops": 4 * rows * case["cols"]}
    if case["kind"] == "norm":          # the stream in, and out where something is added; the addition and the gain in; values and scales out
        stream = 8 if case["add"] else 4
        return {"bytes": rows * (case["cols"] * (stream + size[case["add"]] + 2) + 4) + case["cols"] * size[case["gain"]], "flops": 8 * rows * case["cols"]}
    if case["kind"] == "ffn":           # stream in and out, addition in, result out; the weights and their scales once
        h, f = case["cols"], case["ffn"]
        return {"bytes": rows * h * (8 + 2 * size[case["dtype"]]) + 3 * h * f + 4 * (2 * f + h) + h * size[case["gain"]], "flops": 6 * rows * h * f}
    n, k = case["n"], case["k"]
    out = rows * (n // 2 if case["epilogue"] == "swiglu" else n) * size[case["dtype"]] * (2 if case["epilogue"] == "residual" else 1)
    return {"bytes": (rows + n) * (k + 4) + out, "flops": 2 * rows * n * k}


def _exact_codes(x):
    """In 64 bits: the codes of rows and the scales."""
    top = torch.linalg.vector_norm(x, ord=math.inf, dim=1, keepdim=True)
    return torch.round(x * 127.0 / top), top / 127.0


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "gemm":
        y = torch.mm(s["a"].double(), s["w"].double().T).mul_(torch.outer(s["sa"].double(), s["sw"].double()))
        if case["epilogue"] == "swiglu":
            half = case["n"] // 2
            y = torch.sigmoid(y[:, :half]).mul_(y[:, :half]).mul_(y[:, half:])
        return [y + s["out"].double() if case["epilogue"] == "residual" else y]
    x = s["x"].double()
    if case["kind"] == "quant":
        codes, scale = _exact_codes(x)
        return [scale[:, 0], codes * scale]
    if s["d"] is not None:
        x = x + s["d"].double()
    # the stream is held in fp32: what is normed is the sum rounded to it
    held = x.float().double()
    codes, scale = _exact_codes(held * torch.rsqrt(held.square().sum(1, keepdim=True) / case["cols"] + EPS) * s["gain"].double())
    if case["kind"] == "norm":
        return [x, scale[:, 0], codes * scale]
    y = torch.mm(codes, s["w1"].double().T) * scale * s["sw1"].double()
    f = case["ffn"]
    h = (torch.sigmoid(y[:, :f]) * y[:, :f] * y[:, f:]).to(TORCH[case["dtype"]]).double()
    codes, scale = _exact_codes(h)
    return [x, torch.mm(codes, s["w2"].double().T) * scale * s["sw2"].double()]
