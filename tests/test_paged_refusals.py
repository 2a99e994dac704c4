"""What the operators on a paged cache refuse, through the C ABI, before any HIP call (no GPU needed)."""
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


def shape(**over):
    v = dict(n_seqs=2, n_tokens=5, n_q_heads=8, n_kv_heads=2, page_size=16, n_pages=10, max_pages=4, window=0)
    v.update(over)
    return B.prism_page_shape(*(v[n] for n, _ in B.prism_page_shape._fields_))


def cache(**over):
    v = dict(K=A, V=A, page_stride=2 * 16 * 128, dtype=B.DTYPE_F16, n_kv_heads=2, head_dim=128, page_size=16, n_pages=10)
    v.update(over)
    return B.prism_kv_cache(*(v[n] for n, _ in B.prism_kv_cache._fields_))


BAD_SHAPES = [(dict(n_seqs=-1), B.EINVAL), (dict(n_seqs=4097), B.EINVAL), (dict(n_tokens=-1), B.EINVAL), (dict(n_tokens=1048577), B.EINVAL),
              (dict(n_q_heads=7), B.EINVAL), (dict(n_q_heads=0), B.EINVAL), (dict(n_kv_heads=0), B.EINVAL), (dict(n_q_heads=258), B.EUNSUPPORTED),
              (dict(n_q_heads=514, n_kv_heads=257), B.EUNSUPPORTED), (dict(page_size=8), B.EUNSUPPORTED), (dict(page_size=48), B.EUNSUPPORTED),
              (dict(page_size=512), B.EUNSUPPORTED), (dict(n_pages=0), B.EINVAL), (dict(n_pages=1 << 28), B.EINVAL), (dict(max_pages=0), B.EINVAL),
              (dict(max_pages=(1 << 25) + 1), B.EINVAL), (dict(window=-1), B.EINVAL)]
BAD_CACHES = [(dict(K=0), B.EINVAL), (dict(V=0), B.EINVAL), (dict(V=A + 8), B.EINVAL), (dict(page_stride=2 * 16 * 128 - 8), B.EINVAL),
              (dict(page_stride=2 * 16 * 128 + 4), B.EINVAL), (dict(page_stride=1 << 60), B.EINVAL), (dict(dtype=3), B.EINVAL),
              (dict(head_dim=96), B.EUNSUPPORTED), (dict(head_dim=32), B.EUNSUPPORTED), (dict(head_dim=256), B.EUNSUPPORTED),
              (dict(page_size=24), B.EUNSUPPORTED), (dict(n_pages=0), B.EINVAL), (dict(n_pages=1 << 27), B.EINVAL), (dict(n_kv_heads=0), B.EINVAL)]


def _plan(lib, s=None, **over):
    a = dict(cached=A, fresh=A, table=A, free_pages=A, free_cap=4, n_free=A, left=A, cu=A, pos=A, slot=A, status=A, plan=A)
    a.update(over)
    return lib.prism_op_page_plan(C.byref(s or shape()), *a.values(), None)


@pytest.mark.parametrize("over,code", BAD_SHAPES)
def test_bad_shapes(lib, over, code):
    s = shape(**over)
    assert lib.prism_page_plan_bytes(C.byref(s)) == -1 and lib.prism_attention_paged_workspace(C.byref(s), 128) == -1
    assert _plan(lib, s) == code and lib.prism_last_error()
    assert _attend(lib, s) == code


def test_plan_refuses_missing_and_misaligned_buffers(lib):
    for name in ("cached", "fresh", "table", "free_pages", "n_free", "left", "cu", "pos", "slot", "plan"):
        assert _plan(lib, **{name: None}) == B.EINVAL, name
    assert _plan(lib, plan=A + 8) == B.EINVAL and _plan(lib, free_cap=-1) == B.EINVAL
    assert lib.prism_page_plan_bytes(None) == -1 and lib.prism_attention_paged_workspace(None, 128) == -1


def _finish(lib, c=None, **over):
    a = dict(qkv_dtype=B.DTYPE_FP32, QKV=A, qkv_stride=12 * 128, T=5, pos=A, slot=A, nq=8, q_gain=A, k_gain=A, eps=1e-6, base=1e6, norm=1, Q=A, q_stride=8 * 128)
    a.update(over)
    return lib.prism_op_qkv_finish_paged(C.byref(c or cache()), *a.values(), None)


@pytest.mark.parametrize("over,code", BAD_CACHES)
def test_bad_caches(lib, over, code):
    c = cache(**over)
    assert _finish(lib, c) == code
    assert _attend(lib, None, c) == code


def test_finish_refusals(lib):
    for name in ("QKV", "pos", "slot", "q_gain", "k_gain", "Q"):
        assert _finish(lib, **{name: None}) == B.EINVAL, name
    for over in (dict(T=-1), dict(T=1048577), dict(nq=0), dict(nq=7), dict(base=0.0), dict(qkv_dtype=B.DTYPE_BF16), dict(qkv_stride=12 * 128 - 4),
                 dict(qkv_stride=12 * 128 + 2), dict(q_stride=8 * 128 - 4), dict(q_stride=8 * 128 + 1), dict(QKV=A + 8), dict(Q=A + 4), dict(q_gain=A + 2)):
        assert _finish(lib, **over) == B.EINVAL, over
    assert _finish(lib, T=0, QKV=None) == B.OK


def _attend(lib, s=None, c=None, **over):
    a = dict(plan=A, table=A, Q=A, q_stride=8 * 128, scale=0.0, softcap=0.0, slopes=None, out=A, out_stride=8 * 128, ws=A, ws_bytes=1 << 40)
    a.update(over)
    return lib.prism_op_attention_paged(C.byref(s or shape()), C.byref(c or cache()), *a.values(), None)


def test_attention_refusals(lib):
    for name in ("plan", "table", "Q", "out", "ws"):
        assert _attend(lib, **{name: None}) == B.EINVAL, name
    for over in (dict(plan=A + 4), dict(Q=A + 8), dict(out=A + 2), dict(ws=A + 8), dict(q_stride=8 * 128 - 8), dict(out_stride=8 * 128 + 4), dict(scale=-1.0),
                 dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2e37), dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=2e37),
                 dict(softcap=1e-38), dict(scale=1e10, softcap=1e-30), dict(ws_bytes=100)):
        assert _attend(lib, **over) == B.EINVAL, over
    for over in (dict(n_kv_heads=1, page_stride=16 * 128), dict(page_size=32, page_stride=2 * 32 * 128), dict(n_pages=11)):
        assert _attend(lib, None, cache(**over)) == B.EINVAL, over
    assert _attend(lib, shape(n_tokens=0), plan=None) == B.OK and _attend(lib, shape(n_seqs=0), Q=None) == B.OK
    for hd in (0, -1, 129):
        assert lib.prism_attention_paged_workspace(C.byref(shape()), hd) == -1


def test_sizes_grow_with_the_shape_and_stay_bounded(lib):
    """The workspace is bounded by the number of items wanted, not by the rows; a plan's size is linear in sequences and rows."""
    size = lambda **o: lib.prism_attention_paged_workspace(C.byref(shape(**o)), 128)  # noqa: E731
    assert size(n_tokens=1) < size(n_tokens=100) <= size(n_tokens=10000) == size(n_tokens=1000000) < 1 << 28
    plan = lambda **o: lib.prism_page_plan_bytes(C.byref(shape(**o)))  # noqa: E731
    assert plan(n_tokens=0) < plan(n_tokens=100000) < 1 << 22
