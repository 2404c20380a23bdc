"""Page tables without sequences, and a free list with more places than the pool has pages."""
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


def test_pages_of_the_pool():
    """The list may have more places than the pool has pages, not fewer: a page's number is held against the pool's."""
    table, lens, status = _i32([[0, -1]]), _i32([16]), _i32([0])
    free, n, offs, idx, M = _i32([5, 77, 0, 0, 0, 0, 0, 0]), _i32([2]), _i32([0, 0]), _i32([0] * 8), _i32([0])
    SL.surelock_paged_extend(table, 16, lens, _i32([1]), free, n, offs, idx, M, dev_status=status, n_pages=6)
    assert table.tolist() == [[0, 77]] and status.item() == 4                     # not a page of a pool of 6
    status.zero_()
    SL.surelock_paged_truncate(_i32([[0, 5]]), 16, lens, _i32([0]), free, _i32([0]), dev_status=status, n_pages=6)
    assert free.tolist()[:2] == [0, 5] and status.item() == 0
    few = _i32([5, 3])
    with pytest.raises(SL.SurelockError):
        SL.surelock_paged_extend(table, 16, lens, _i32([1]), few, n, offs, idx, M, n_pages=6)
    with pytest.raises(SL.SurelockError):
        SL.surelock_paged_truncate(table, 16, lens, _i32([0]), few, n, n_pages=6)
