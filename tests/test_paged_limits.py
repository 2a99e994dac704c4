"""Limits of the operators on a paged cache: the largest launch, the furthest position."""
import ctypes as C

import numpy as np
import pytest
import torch

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


@pytest.mark.gpu
def test_positions_beyond_the_furthest():
    """More than 2^29 cached tokens count as 2^29: behind every table's end."""
    ints = lambda a: torch.as_tensor(np.asarray(a, np.int32)).to("cuda")  # noqa: E731
    cached, fresh = [2 ** 29 - 1, 2 ** 29, 2 ** 29 + 1, 2 ** 31 - 1], [3, 2, 2, 1]
    plan = B.PagePlan(4, 9, 8, 2, 16, 40, 3)
    table, left, cu, pos, slot, status = (ints(x) for x in (np.full((4, 3), 7), [0], [0] * 5, [0] * 9, [0] * 9, [0] * 4))
    B.op_page_plan(plan, ints(cached), ints(fresh), table, ints([1, 2, 3]), ints([3]), left, cu, pos, slot, status)
    far = 2 ** 29
    assert pos.tolist() == [far - 1, far, far + 1, far, far + 1, far, far + 1, far, 0] and slot.tolist() == [-1] * 9
    assert cu.tolist() == [0, 3, 5, 7, 8] and status.tolist() == [8, 0, 0, 0] and left.tolist() == [3] and (table == 7).all()
