"""Page tables, row offsets and flat positions from request lengths: whole numbers, compared for equality with a loop over the
sequences."""
import ctypes

import pytest
import torch

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import build as build_mod

DEV = "cuda"
gpu = pytest.mark.gpu


def _ceil(a, b):
    return -(-a // b)


def extend(table, P, lens, new, free, n_free, rows):
    """The definition: (table, lens, n_free, offsets, idx)."""
    table, lens = [list(r) for r in table], list(lens)
    W = len(table[0])
    top, wanted, wanted_rows, offs, idx = n_free, 0, 0, [0], []
    for b in range(len(lens)):
        if lens[b] + new[b] <= W * P:
            need = _ceil(lens[b] + new[b], P) - _ceil(lens[b], P)
            wanted, wanted_rows = wanted + need, wanted_rows + new[b]
            if (need == 0 or wanted <= n_free) and wanted_rows <= rows:
                for j in range(_ceil(lens[b], P), _ceil(lens[b] + new[b], P)):
                    top -= 1
                    table[b][j] = free[top]
                idx += [b * W * P + lens[b] + i for i in range(new[b])]
                lens[b] += new[b]
        offs.append(len(idx))
    return table, lens, top, offs, idx


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Plan:
    def __init__(self, B, W, P, n_pages, lens, seed=0):
        g = torch.Generator().manual_seed(seed)
        order = torch.randperm(n_pages, generator=g).tolist()
        self.P, self.W, self.B, self.n_pages = P, W, B, n_pages
        self.lens = list(lens)
        self.table = [[-1] * W for _ in range(B)]
        for b in range(B):
            for j in range(_ceil(lens[b], P)):
                self.table[b][j] = order.pop()
        self.free, self.n_free = order + [-7] * (n_pages - len(order)), len(order)

    def extend(self, new, rows, in_place=True):
        t, l, f, n = _i32(self.table), _i32(self.lens), _i32(self.free), _i32([self.n_free])
        idx, offs, M, status = _i32([-5] * rows), _i32([-5] * (self.B + 1)), _i32([-5]), _i32([0])
        lo, no = (l, n) if in_place else (_i32([-5] * self.B), _i32([-5]))
        SL.surelock_paged_extend(t, self.P, l, _i32(new), f, n, offs, idx, M, None if in_place else lo, None if in_place else no, status)
        want = extend(self.table, self.P, self.lens, new, self.free, self.n_free, rows)
        assert f.tolist() == self.free and status.item() == 0
        if not in_place:
            assert l.tolist() == self.lens and n.tolist() == [self.n_free]
        assert (t.tolist(), lo.tolist(), no.item(), offs.tolist(), idx.tolist()[:M.item()]) == want
        assert M.item() == want[3][-1] and idx.tolist()[M.item():] == [-5] * (rows - M.item())
        self.table, self.lens, self.n_free = want[:3]
        return want[3], want[4]

    def truncate(self, keep, in_place=True):
        t, l, f, n, status = _i32(self.table), _i32(self.lens), _i32(self.free), _i32([self.n_free]), _i32([0])
        lo, no = (l, n) if in_place else (_i32([-5] * self.B), _i32([-5]))
        SL.surelock_paged_truncate(t, self.P, l, _i32(keep), f, n, None if in_place else lo, None if in_place else no, status)
        for b in range(self.B):
            k = min(keep[b], self.lens[b])
            for j in range(_ceil(k, self.P), _ceil(self.lens[b], self.P)):
                self.free[self.n_free] = self.table[b][j]
                self.n_free += 1
            self.lens[b] = k
        assert t.tolist() == self.table and lo.tolist() == self.lens and f.tolist() == self.free
        assert no.item() == self.n_free and status.item() == 0


# ---- refusals, without a GPU ------------------------------------------------------------------------------------------
def test_refusals_on_the_host():
    build_mod.build()
    L = SL.lib()
    good = [0x100, 4, 64, 8, 100, 0x200, 0x300, 0x400, 0x500, 0x600, 0x700, 0x800, 10, 0x900, 0xa00, None, None]
    for at, value, rc in [(0, None, -1), (1, 0, -1), (2, 0, -5), (2, 48, -5), (2, 512, -5), (3, 0, -1), (4, 0, -1), (5, None, -1), (6, None, -1), (7, None, -1),
                          (8, None, -1), (9, None, -1), (10, None, -1), (11, None, -1), (12, -1, -1), (13, None, -1), (14, None, -1), (1, 1025, -5),
                          (3, 1 << 23, -5)]:
        bad = list(good)
        bad[at] = value
        assert L.surelock_paged_extend(*bad) == rc, (at, value)
    good = [0x100, 4, 64, 8, 100, 0x200, 0x300, 0x400, 0x500, 0x600, 0x700, None, None]
    for at, value, rc in [(0, None, -1), (1, 0, -1), (1, 1025, -5), (2, 17, -5), (3, -1, -1), (4, -1, -1), (5, None, -1), (6, None, -1), (7, None, -1), (8, None, -1),
                          (9, None, -1), (10, None, -1), (3, 1 << 23, -5)]:
        bad = list(good)
        bad[at] = value
        assert L.surelock_paged_truncate(*bad) == rc, (at, value)


def test_binding_refuses_tensors_of_the_host():
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(SL.SurelockError):
        SL.surelock_paged_extend(torch.zeros(2, 2, dtype=torch.int32), 64, z, z, z, z, z, z, z)
    with pytest.raises(SL.SurelockError):
        SL.surelock_paged_truncate(torch.zeros(2, 2, dtype=torch.int32), 64, z, z, z, z)


# ---- on the GPU -------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("B,W,P,n_pages,rows", [(1, 1, 16, 1, 16), (3, 5, 16, 9, 100), (32, 64, 64, 700, 32), (128, 9, 32, 600, 4096),
                                                (129, 9, 32, 600, 4097), (1000, 40, 16, 9000, 30000), (1024, 3, 256, 3000, 200000)])
@pytest.mark.parametrize("in_place", [True, False])
def test_a_batch_grows_and_shrinks(B, W, P, n_pages, rows, in_place):
    """Prompts, single tokens, more than there are pages or rows for, requests that end: each call against the loop."""
    g = torch.Generator().manual_seed(B + rows)
    r = lambda hi, n=B: torch.randint(0, hi + 1, (n,), generator=g).tolist()
    plan = Plan(B, W, P, n_pages, [0] * B)
    plan.extend(r(min(W * P, 2 * P)), rows, in_place)
    plan.extend([1] * B, rows, in_place)
    plan.extend([0] * B, rows, in_place)
    plan.truncate([n - 1 if n % 3 else n + 5 for n in plan.lens] if min(plan.lens) else [max(0, n - 1) for n in plan.lens], in_place)
    plan.extend(r(W * P + 3), rows, in_place)                     # some pass their table
    plan.extend(r(3 * P), rows, in_place)
    plan.truncate(r(W * P), in_place)
    plan.extend(r(P), rows, in_place)
    plan.truncate([0] * B, in_place)
    assert plan.n_free == n_pages and sorted(plan.free) == list(range(n_pages))


@gpu
def test_borders():
    """The last page, the last row, the last place of a table; a sequence that needs no page is served when the list is empty."""
    plan = Plan(4, 2, 16, 4, [15, 16, 0, 31])                     # 1 + 1 + 0 + 2 pages: the list is empty
    assert plan.n_free == 0
    assert plan.extend([1, 1, 0, 1], 8)[0] == [0, 1, 1, 1, 2]     # the second needs a page, the last one does not
    plan.truncate([0, 16, 0, 32])
    assert plan.n_free == 1
    assert plan.extend([16, 1, 0, 0], 16)[0] == [0, 16, 16, 16, 16]       # rows for the first only
    plan.truncate([0, 16, 0, 32])
    assert plan.extend([17, 16, 0, 0], 100)[0] == [0, 0, 0, 0, 0]         # two pages wanted by the first: nobody behind it overtakes
    assert plan.extend([33, 16, 0, 0], 100)[0] == [0, 0, 16, 16, 16]      # one that fits no table does not hold the others up
    assert plan.extend([0, 0, 0, 0], 0)[0] == [0, 0, 0, 0, 0]


@gpu
def test_bad_numbers_are_clamped_and_reported():
    for lens, new, n_free, want in [([3, 5], [-4, 1], 4, ([3, 6], [0, 0, 1])), ([-2, 5], [1, 0], 4, ([1, 5], [0, 1, 1])), ([3, 99], [0, 0], 4, ([3, 32], [0, 0, 0])),
                                    ([3, 5], [0, 0], 9, ([3, 5], [0, 0, 0])), ([3, 5], [14, 0], -1, ([3, 5], [0, 0, 0]))]:
        table, l, free, n = _i32([[0, -1], [1, -1]]), _i32(lens), _i32([2, 3, 4, 5]), _i32([n_free])
        offs, idx, M, status = _i32([0] * 3), _i32([0] * 50), _i32([0]), _i32([0])
        SL.surelock_paged_extend(table, 16, l, _i32(new), free, n, offs, idx, M, dev_status=status)
        assert (l.tolist(), offs.tolist()) == want and status.item() == 4
    # a page outside the pool is passed on and reported; more pages than the list has places are dropped
    table, l, n, offs, idx, M, status = _i32([[0, -1]]), _i32([16]), _i32([1]), _i32([0] * 2), _i32([0] * 9), _i32([0]), _i32([0])
    SL.surelock_paged_extend(table, 16, l, _i32([3]), _i32([77, 1]), n, offs, idx, M, dev_status=status)
    assert table.tolist() == [[0, 77]] and status.item() == 4
    free, n, l, status = _i32([1, 0, 9]), _i32([2]), _i32([32]), _i32([0])
    SL.surelock_paged_truncate(_i32([[2, 1]]), 16, l, _i32([0]), free, n, dev_status=status)
    assert free.tolist() == [1, 0, 2] and n.item() == 3 and l.item() == 0 and status.item() == 4


@gpu
def test_replayed_with_other_lengths():
    B, W, P, rows = 40, 8, 16, 5000
    n_pages = B * W
    t, l, new, f, n = _i32([[-1] * W] * B), _i32([0] * B), _i32([1] * B), _i32(list(range(n_pages))), _i32([n_pages])
    offs, idx, M = _i32([0] * (B + 1)), _i32([0] * rows), _i32([0])
    SL.surelock_paged_extend(t, P, l, new, f, n, offs, idx, M)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        SL.surelock_paged_extend(t, P, l, new, f, n, offs, idx, M)
    table, lens, top = [list(r) for r in t.tolist()], l.tolist(), n.item()
    for seed in range(6):
        take = torch.randint(0, 30, (B,), generator=torch.Generator().manual_seed(seed)).tolist()
        new.copy_(_i32(take))
        graph.replay()
        table, lens, top, want_offs, want_idx = extend(table, P, lens, take, f.tolist(), top, rows)
        assert (t.tolist(), l.tolist(), n.item(), offs.tolist(), idx.tolist()[:M.item()]) == (table, lens, top, want_offs, want_idx)
