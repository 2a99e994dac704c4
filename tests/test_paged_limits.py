"""Limits of the operators on a paged cache: the largest launch."""
import ctypes as C

import pytest

from paper_2510_15620_amd import binding as B

A = 1 << 20          # an address that is aligned and never followed


@pytest.mark.parametrize("n_tokens,nq,nkv", [(1048576, 128 * 17, 17), (1048576, 128 * 256, 256), (600000, 65 * 32, 32)])
def test_more_workgroups_than_a_launch_can_have(n_tokens, nq, nkv):
    """2^32 threads are the most that a launch may have: 2^24 workgroups, one for each work item and KV head."""
    s = B.prism_page_shape(2, n_tokens, nq, nkv, 16, 10, 4, 0)
    c = B.prism_kv_cache(A, A, nkv * 16 * 64, B.DTYPE_F16, nkv, 64, 16, 10)
    lib = B.lib()
    code = lib.prism_op_attention_paged(C.byref(s), C.byref(c), A, A, A, nq * 64, 0.0, 0.0, None, A, nq * 64, A, 1 << 50, None)
    assert code == B.EUNSUPPORTED and b"work items" in lib.prism_last_error()
