"""What the operators on 8-bit rows refuse, through the C ABI, before any HIP call (no GPU needed)."""
import ctypes as C
import os

import pytest

from paper_2510_15620_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2510_15620_amd import build
        build.build(verbose=False)
    return B.lib()


A = 1 << 20          # an address that is aligned and never followed
MAX = 1 << 23


def rows(**over):
    v = dict(codes=A, scales=A, stride=256, rows=5, cols=200)
    v.update(over)
    return B.prism_q8(*(v[n] for n, _ in B.prism_q8._fields_))


def quantize(lib, q=None, **over):
    a = dict(dtype=B.DTYPE_F16, X=A, x_stride=200)
    a.update(over)
    return lib.prism_op_quantize_q8(*a.values(), C.byref(q or rows()), None)


def dequantize(lib, q=None, **over):
    a = dict(dtype=B.DTYPE_BF16, out=A, out_stride=200)
    a.update(over)
    return lib.prism_op_dequantize_q8(C.byref(q or rows()), *a.values(), None)


def norm(lib, q=None, **over):
    a = dict(X=A, x_stride=200, add_dtype=B.DTYPE_F16, add=A, add_stride=200, gain_dtype=B.DTYPE_BF16, gain=A, eps=1e-6)
    a.update(over)
    return lib.prism_op_rmsnorm_q8(*a.values(), C.byref(q or rows()), None)


def gemm(lib, a=None, w=None, **over):
    v = dict(dtype=B.DTYPE_F16, out=A, out_stride=60)
    v.update(over)
    epilogue = v.pop("epilogue", B.EPI_STORE)
    return lib.prism_op_gemm_q8(epilogue, C.byref(a or rows()), C.byref(w or rows(rows=60)), *v.values(), None)


BAD_ROWS = [dict(codes=0), dict(scales=0), dict(codes=A + 8), dict(scales=A + 2), dict(stride=240), dict(stride=264), dict(stride=MAX + 16), dict(rows=-1),
            dict(rows=1048577), dict(cols=0), dict(cols=-4), dict(cols=131072, stride=131072)]


@pytest.mark.parametrize("over", BAD_ROWS)
def test_bad_rows(lib, over):
    q = rows(**over)
    wide = dict(x_stride=1 << 20) if over.get("cols", 0) > 200 else {}
    assert quantize(lib, q, **wide) == B.EINVAL and lib.prism_last_error()
    assert dequantize(lib, q) == B.EINVAL and norm(lib, q) == B.EINVAL
    assert gemm(lib, q) == B.EINVAL and gemm(lib, None, q) == B.EINVAL


def test_missing_rows(lib):
    assert lib.prism_op_quantize_q8(B.DTYPE_F16, A, 200, None, None) == B.EINVAL
    assert lib.prism_op_dequantize_q8(None, B.DTYPE_F16, A, 200, None) == B.EINVAL
    assert lib.prism_op_rmsnorm_q8(A, 200, 0, None, 0, 0, A, 1e-6, None, None) == B.EINVAL
    assert lib.prism_op_gemm_q8(B.EPI_STORE, None, C.byref(rows()), B.DTYPE_F16, A, 60, None) == B.EINVAL
    assert lib.prism_op_gemm_q8(B.EPI_STORE, C.byref(rows()), None, B.DTYPE_F16, A, 60, None) == B.EINVAL


def test_quantize_and_dequantize_refusals(lib):
    for over in (dict(dtype=3), dict(dtype=-1), dict(x_stride=199), dict(x_stride=MAX + 1), dict(X=None), dict(X=A + 1)):
        assert quantize(lib, **over) == B.EINVAL, over
    for over in (dict(dtype=3), dict(out_stride=199), dict(out_stride=MAX + 1), dict(out=None), dict(out=A + 1)):
        assert dequantize(lib, **over) == B.EINVAL, over
    assert quantize(lib, dtype=B.DTYPE_FP32, X=A + 2) == B.EINVAL and dequantize(lib, dtype=B.DTYPE_FP32, out=A + 2) == B.EINVAL
    none = rows(rows=0, codes=0, scales=0)
    assert quantize(lib, none, X=None) == B.OK and dequantize(lib, none, out=None) == B.OK


def test_norm_refusals(lib):
    for over in (dict(X=None), dict(gain=None), dict(X=A + 2), dict(add=A + 1), dict(gain=A + 1), dict(add_dtype=3), dict(gain_dtype=3), dict(gain_dtype=-1), dict(x_stride=199),
                 dict(add_stride=199), dict(x_stride=MAX + 1), dict(add_stride=MAX + 1), dict(eps=0.0), dict(eps=-1e-6), dict(eps=float("nan")), dict(eps=float("inf")),
                 dict(add_dtype=B.DTYPE_FP32, add=A + 2), dict(gain_dtype=B.DTYPE_FP32, gain=A + 2)):
        assert norm(lib, **over) == B.EINVAL, over
    assert norm(lib, rows(rows=0), X=None) == B.OK


def test_gemm_refusals(lib):
    for over in (dict(epilogue=4), dict(epilogue=-1), dict(dtype=B.DTYPE_FP32), dict(dtype=3), dict(epilogue=B.EPI_SWIGLU, dtype=B.DTYPE_FP32),
                 dict(epilogue=B.EPI_RESIDUAL), dict(epilogue=B.EPI_STORE_F32, dtype=B.DTYPE_BF16), dict(out_stride=59), dict(out_stride=MAX + 1), dict(out=None), dict(out=A + 1),
                 dict(epilogue=B.EPI_STORE_F32, dtype=B.DTYPE_FP32, out=A + 2)):
        assert gemm(lib, **over) == B.EINVAL, over
    assert gemm(lib, rows(cols=199)) == B.EINVAL                                   # rows of different lengths
    assert gemm(lib, None, rows(rows=61), epilogue=B.EPI_SWIGLU) == B.EUNSUPPORTED
    assert gemm(lib, None, rows(rows=1 << 20, stride=4096), out_stride=1 << 20) == B.EUNSUPPORTED       # 4 GiB of weights
    assert gemm(lib, rows(rows=0), out=None) == B.OK and gemm(lib, None, rows(rows=0), out=None) == B.OK
