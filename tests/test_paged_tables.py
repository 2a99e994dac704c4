"""Page tables whose rows are not those of the plan are refused (no GPU needed: the check looks at the tensor only)."""
import pytest
import torch

from paper_2510_15620_amd import binding as B


@pytest.fixture
def torch_known(monkeypatch):
    monkeypatch.setattr(B, "_torch", torch)


def _plan(n_seqs, max_pages):
    plan = B.PagePlan.__new__(B.PagePlan)
    plan.n_seqs, plan.max_pages = n_seqs, max_pages
    return plan


@pytest.mark.parametrize("shape", [(3, 8), (4, 8), (24,), (30,), (1, 3, 8)])
def test_tables_that_fit(torch_known, shape):
    t = torch.zeros(shape, dtype=torch.int32)
    assert B._table(t, _plan(3, 8), -1) == t.data_ptr()


@pytest.mark.parametrize("shape", [(3, 9), (3, 16), (4, 6), (24, 1), (6, 4), (2, 8), (23,), (8, 3), (3, 8, 1)])
def test_tables_with_other_rows(torch_known, shape):
    with pytest.raises(B.PrismError) as e:
        B._table(torch.zeros(shape, dtype=torch.int32), _plan(3, 8), -1)
    assert e.value.code == B.EINVAL


def test_tables_of_other_types_or_strides(torch_known):
    for t in (torch.zeros(3, 8, dtype=torch.int64), torch.zeros(3, 16, dtype=torch.int32)[:, :8], torch.zeros(8, 3, dtype=torch.int32).T):
        with pytest.raises(B.PrismError):
            B._table(t, _plan(3, 8), -1)
    with pytest.raises(B.PrismError):
        B._table(torch.zeros(3, 8, dtype=torch.int32), _plan(3, 8), 0)


@pytest.mark.gpu
def test_calls_with_a_table_of_longer_rows():
    from tests import paged_reference as R
    s = R.Step([20, 70], [3, 1], 16, 4, 2, 64, torch.float16)
    out = s.make_plan()
    wide = torch.full((2, s.table.shape[1] + 3), -1, dtype=torch.int32, device="cuda")
    wide[:, : s.table.shape[1]] = s.device(s.table)
    before = wide.clone()
    with pytest.raises(B.PrismError) as e:
        B.op_page_plan(s.plan, s.device(s.cached), s.device(s.fresh), wide, s.device(s.free), s.device([len(s.free)]), out["left"], out["cu"], out["pos"], out["slot"])
    assert e.value.code == B.EINVAL and torch.equal(wide, before)
    o = torch.full_like(s.Q, 7.0)
    with pytest.raises(B.PrismError) as e:
        B.op_attention_paged(s.plan, s.Q, s.cache, wide, o, B.attention_paged_workspace(s.plan, s.cache))
    assert e.value.code == B.EINVAL and (o == 7).all()
    B.op_attention_paged(s.plan, s.Q, s.cache, s.d_table.view(-1), o, B.attention_paged_workspace(s.plan, s.cache))
    assert torch.equal(o, s.check())
