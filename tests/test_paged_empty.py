"""Page tables without sequences."""
import pytest
import torch

from paper_2602_06412_b200 import binding as SL

from .test_paged_plan import _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [True, False])
def test_an_empty_batch(in_place):
    """No rows, nothing taken: what was in the outputs before does not stay as if it were this call's."""
    none, free, n, status = _i32([]), _i32([5, 2, 7]), _i32([2]), _i32([0])
    offs, idx, M, out = _i32([9]), _i32([8, 8]), _i32([9]), None if in_place else _i32([9])
    table = torch.zeros(0, 4, dtype=torch.int32, device="cuda")
    SL.surelock_paged_extend(table, 16, none, none, free, n, offs, idx, M, n_free_out=out, dev_status=status)
    assert offs.tolist() == [0] and M.item() == 0 and idx.tolist() == [8, 8] and (n if in_place else out).item() == 2
    out = None if in_place else _i32([9])
    SL.surelock_paged_truncate(table, 16, none, none, free, n, n_free_out=out, dev_status=status)
    assert free.tolist() == [5, 2, 7] and n.item() == 2 and (n if in_place else out).item() == 2 and status.item() == 0
