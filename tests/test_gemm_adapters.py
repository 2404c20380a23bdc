"""Low-rank adapters beside a projection, against a statement in 64 bits.

With small whole numbers and scale 1 every product and sum is exact in fp32, so an fp32 C is compared for equality: that pins every
index.  With random values the bound follows the roundings: t = A x is a chain of at most K / 16 matrix instructions and 64 partial
sums, each off by at most 2^-22 of sum |a| |x|; t scale enters the second product to 2^-24 of itself (bf16 C: 2^-17), whose at most
24 instructions are off by 2^-22 of sum |b| |t| each; then C's own rounding, 2^-24 or 2^-8 of it, after an fp32 addition."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import build as build_mod

DEV = "cuda"
gpu = pytest.mark.gpu


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _make(n_ad, rank, K, n_out, seed, exact=False):
    g = torch.Generator().manual_seed(seed)
    if exact:
        a, b = torch.randint(-2, 3, (n_ad, rank, K), generator=g), torch.randint(-2, 3, (n_ad, n_out, rank), generator=g)
        scale = torch.exp2(torch.randint(-1, 2, (n_ad,), generator=g).float())
    else:
        a, b, scale = torch.randn(n_ad, rank, K, generator=g) * K ** -0.5, torch.randn(n_ad, n_out, rank, generator=g) * 0.2, torch.randn(n_ad, generator=g) * 2
    return a.to(torch.bfloat16), b.to(torch.bfloat16), scale.float()


def _want(x, c, a, b, scale, ranks, which, offs):
    """(result, tolerance but for C's own rounding) in 64 bits."""
    x, c, a, b, scale = (t.double().numpy() for t in (x, c, a, b, scale))
    y, tol = c.copy(), np.zeros_like(c)
    K = x.shape[1]
    for s, ad in enumerate(which):
        if ad < 0:
            continue
        rows, r = slice(offs[s], offs[s + 1]), ranks[ad]
        t, size = x[rows] @ a[ad, :r].T, np.abs(x[rows]) @ np.abs(a[ad, :r]).T
        bt, sc = b[ad, :, :r].T, abs(scale[ad])
        y[rows] += scale[ad] * (t @ bt)
        tol[rows] = sc * ((K / 16 + 64) * 2.0 ** -22 * (size @ np.abs(bt)) + 24 * 2.0 ** -22 * (np.abs(t) @ np.abs(bt)))
        tol[rows] += sc * 2.0 ** -24 * (np.abs(t) @ np.abs(bt))
    return y, tol


def _rows(B, kind, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        return [1] * B
    if kind == "some":
        return torch.randint(0, 5, (B,), generator=g).tolist()
    return torch.randint(0, int(kind) + 1, (B,), generator=g).tolist()


# ---- refusals, without a GPU ------------------------------------------------------------------------------------------
def test_refusals_on_the_host():
    build_mod.build()
    L = SL.lib()
    w = lambda **o: ctypes.byref(SL._Adapters(**{**dict(a=0x1000, b=0x2000, scale=0x3000, ranks=None, n_adapters=4, max_rank=16), **o}))
    good = [0x100, w(), 0x200, 0x300, 3, 0x400, 100, 5, 100, 64, SL.SL_BF16, None, None]
    for at, value, rc in [(0, None, -1), (1, None, -1), (1, w(a=None), -1), (1, w(b=None), -1), (1, w(scale=None), -1), (1, w(n_adapters=0), -1), (1, w(max_rank=0), -1),
                          (2, None, -1), (3, None, -1), (4, 0, -1), (5, None, -1), (6, 99, -1), (7, -1, -1), (8, 0, -1), (9, 0, -1), (10, SL.SL_INT8, -1), (9, 60, -5),
                          (1, w(max_rank=12), -5), (1, w(max_rank=136), -5), (0, 0x108, -5), (1, w(a=0x1008), -5), (1, w(b=0x2008), -5), (5, 0x401, -5), (7, 0, 0)]:
        bad = list(good)
        bad[at] = value
        assert L.surelock_gemm_adapters(*bad) == rc, (at, value)


# ---- on the GPU -------------------------------------------------------------------------------------------------------
SHAPES = [(1, "one", 1, 16, 4096, 4096), (5, "some", 3, 8, 64, 40), (64, "one", 9, 64, 1024, 520), (70, "some", 7, 24, 200, 33), (3, "200", 4, 32, 520, 96),
          (9, "90", 5, 128, 1032, 257), (2, "700", 2, 16, 96, 1000), (4, "130", 3, 56, 8, 5), (300, "one", 20, 16, 512, 64), (1, "4000", 1, 40, 256, 128),
          (7, "one", 4, 104, 264, 77), (20, "some", 6, 48, 1160, 161), (6, "20", 3, 120, 136, 1001),
          # many rows to a sequence and rank enough for the kernel that takes 128 at a time
          (3, "2500", 4, 32, 520, 96), (9, "400", 5, 128, 1032, 257), (2, "6000", 2, 16, 96, 1000), (4, "900", 3, 56, 8, 5), (5, "300", 2, 72, 200, 64)]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,kind,n_ad,rank,K,n_out", SHAPES)
def test_random_values(dtype, B, kind, n_ad, rank, K, n_out):
    """Ranks of their own (what lies behind them is NaN), requests without an adapter or rows, C a part of wider rows."""
    g = torch.Generator().manual_seed(B + rank)
    counts = _rows(B, kind, 3)
    M, spare = sum(counts), 3
    offs = [0] + np.cumsum(counts).tolist()
    a, b, scale = _make(n_ad, rank, K, n_out, 5)
    ranks = torch.randint(0, rank + 1, (n_ad,), generator=g).tolist()
    ranks[0] = rank
    for i, r in enumerate(ranks):
        a[i, r:], b[i, :, r:] = float("nan"), float("nan")
    which = torch.randint(-1, n_ad, (B,), generator=g).tolist()
    which[0] = 0
    x = torch.randn(M + spare, K, generator=g).to(torch.bfloat16)
    wide = torch.randn(M + spare, n_out + 24, generator=g).to(dtype)
    c = wide.to(DEV)
    status = _i32([0])
    SL.surelock_gemm_adapters(x.to(DEV), SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV), _i32(ranks)), _i32(which), _i32(offs), c[:, 8:8 + n_out], status)
    want, tol = _want(x, wide[:, 8:8 + n_out], a, b, scale, ranks, which, offs)
    if dtype == torch.bfloat16:                                    # t as a number of 17 bits
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -17 * np.abs(want - wide[:, 8:8 + n_out].double().numpy()) + 0
        extra = np.zeros_like(tol)
        for s, ad in enumerate(which):
            if ad >= 0:
                rows, r = slice(offs[s], offs[s + 1]), ranks[ad]
                t = np.abs(x[rows].double().numpy() @ a[ad, :r].double().numpy().T)
                extra[rows] = 2.0 ** -17 * abs(scale[ad].item()) * (t @ np.abs(b[ad, :, :r].double().numpy()).T)
        tol = tol + extra
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    got = c[:, 8:8 + n_out].cpu().double().numpy()
    assert np.all(np.abs(got - want) <= tol + half * np.abs(want) + 2.0 ** -24 * (np.abs(want) + tol))
    untouched = torch.ones_like(wide, dtype=torch.bool)
    for s, ad in enumerate(which):
        if ad >= 0 and ranks[ad]:
            untouched[offs[s]:offs[s + 1], 8:8 + n_out] = False
    assert torch.equal(c.cpu()[untouched], wide[untouched]) and status.item() == 0


@gpu
@pytest.mark.parametrize("B,kind,n_ad,rank,K,n_out", SHAPES)
def test_whole_numbers_are_exact(B, kind, n_ad, rank, K, n_out):
    g = torch.Generator().manual_seed(B)
    counts = _rows(B, kind, 4)
    M, offs = sum(counts), [0] + np.cumsum(counts).tolist()
    a, b, scale = _make(n_ad, rank, K, n_out, 6, exact=True)
    which = torch.randint(0, n_ad, (B,), generator=g).tolist()
    x = torch.randint(-2, 3, (max(M, 1), K), generator=g).to(torch.bfloat16)
    c0 = torch.randint(-9, 10, (max(M, 1), n_out), generator=g).float()
    c = c0.to(DEV)
    SL.surelock_gemm_adapters(x.to(DEV), SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV)), _i32(which), _i32(offs), c)
    want, _ = _want(x, c0, a, b, scale, [rank] * n_ad, which, offs)
    assert np.abs(want).max() < 2 ** 23 and np.array_equal(c.cpu().double().numpy(), want)


@gpu
def test_a_row_does_not_touch_others_and_special_values_pass():
    a, b, scale = _make(2, 16, 128, 64, 7)
    x = torch.randn(20, 128, generator=torch.Generator().manual_seed(7)).to(torch.bfloat16)
    x[4, 9], x[11, 0] = float("nan"), float("inf")
    ad = SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV))
    c = torch.zeros(20, 64, device=DEV)
    SL.surelock_gemm_adapters(x.to(DEV), ad, _i32([0, 1]), _i32([0, 13, 20]), c)
    bad = ~torch.isfinite(c).cpu()
    assert bad[4].all() and bad[11].any() and not bad[[r for r in range(20) if r not in (4, 11)]].any()
    assert torch.isnan(c[4]).all()


@gpu
def test_bad_numbers_are_reported():
    a, b, scale = _make(2, 16, 64, 32, 8)
    x, c0 = torch.randn(6, 64).to(torch.bfloat16).to(DEV), torch.randn(6, 32, device=DEV)
    for which, offs, ranks in [([0, 2], [0, 3, 6], None), ([0, 1], [0, 3, 9], None), ([0, 1], [-2, 3, 6], None), ([0, 0], [0, 3, 6], [17, 3]), ([0, 0], [0, 3, 6], [-1, 3])]:
        c, status = c0.clone(), _i32([0])
        SL.surelock_gemm_adapters(x, SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV), None if ranks is None else _i32(ranks)), _i32(which), _i32(offs), c, status)
        assert status.item() == 4
        if which[1] == 2:
            assert torch.equal(c[3:], c0[3:])


@gpu
@pytest.mark.parametrize("B,rows,cap", [(8, 1, 8), (3, 70, 400), (3, 500, 1600)])
def test_replayed_with_other_requests_and_deterministic(B, rows, cap):
    a, b, scale = _make(6, 32, 256, 160, 9)
    ad = SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV))
    x = torch.randn(cap, 256, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    c0 = torch.randn(cap, 160, generator=torch.Generator().manual_seed(10))
    xd, c, which, offs = x.to(DEV), c0.to(DEV), _i32([0] * B), _i32([0] * (B + 1))
    SL.surelock_gemm_adapters(xd, ad, which, offs, c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        SL.surelock_gemm_adapters(xd, ad, which, offs, c)
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        counts = torch.randint(0, rows + 1, (B,), generator=g).tolist()
        o, w = [0] + np.cumsum(counts).tolist(), torch.randint(-1, 6, (B,), generator=g).tolist()
        which.copy_(_i32(w))
        offs.copy_(_i32(o))
        out = []
        for _ in range(2):
            c.copy_(c0)
            graph.replay()
            out.append(c.clone())
        want, tol = _want(x, c0, a, b, scale, [32] * 6, w, o)
        assert np.all(np.abs(out[0].cpu().double().numpy() - want) <= tol + 2.0 ** -23 * np.abs(want)) and torch.equal(*out)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rank,K,rows", [(16, 1024, 3200), (128, 320, 700)])
def test_a_lost_copy_ends_the_call_with_a_status(dtype, rank, K, rows):
    """The bounded waits run out: status 2, the tile's rows are NaN, the others right, and so is the next call."""
    a, b, scale = _make(2, rank, K, 300, 11)
    ad = SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV))
    x = torch.randn(rows, K, generator=torch.Generator().manual_seed(11)).to(torch.bfloat16).to(DEV)
    c0 = torch.randn(rows, 300, generator=torch.Generator().manual_seed(12)).to(dtype).to(DEV)
    which, offs, status = _i32([0, 1]), _i32([0, 400, rows]), _i32([0])
    run = lambda: (lambda c: (SL.surelock_gemm_adapters(x, ad, which, offs, c, status), c)[1])(c0.clone())
    want = run()
    assert status.item() == 0
    SL.surelock_lose_next_copy()
    got = run()
    assert status.item() == 2 and bool(torch.isnan(got[:128]).all()) and torch.equal(got[128:], want[128:])
    status.zero_()
    assert torch.equal(run(), want) and status.item() == 0


@gpu
def test_no_wait_runs_to_its_limit_when_a_kernel_leaves():
    """Before a CTA leaves it waits for its copies and products, at most 2 s and without a status: a wait for the wrong phase would
    show as time only.  Numbers of blocks of k and of features below, at and above the rings' sizes."""
    import time
    for K in (8, 64, 72, 192, 256, 520, 1104):
        for n_out in (5, 64, 130, 260, 700):
            for rank in (16, 128):
                a, b, scale = _make(1, rank, K, n_out, 13)
                ad = SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV))
                rows = 3200 if rank == 16 else 400
                x = torch.zeros(rows, K, dtype=torch.bfloat16, device=DEV)
                for dtype in (torch.bfloat16, torch.float32):
                    c = torch.zeros(rows, n_out, dtype=dtype, device=DEV)
                    torch.cuda.synchronize()
                    t = time.perf_counter()
                    SL.surelock_gemm_adapters(x, ad, _i32([0]), _i32([0, rows]), c)
                    torch.cuda.synchronize()
                    assert time.perf_counter() - t < 1.0


@gpu
@pytest.mark.parametrize("rows,n_out,pitch,offset", [(2200, 96, 96, 0), (2200, 96, 104, 8), (2200, 96, 97, 1), (2200, 95, 96, 0), (40, 33, 40, 3), (300, 64, 1000, 936),
                                                       (2100, 64, 1000, 936), (2100, 100, 104, 0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_outputs_anywhere(dtype, rows, n_out, pitch, offset):
    """C in wider rows, off 16 bytes, with a last tile that is not whole: the neighbours of every row stay as they are."""
    a, b, scale = _make(2, 24, 256, n_out, 14, exact=True)
    x = torch.randint(-2, 3, (rows, 256), generator=torch.Generator().manual_seed(14)).to(torch.bfloat16)
    flat = torch.randint(-9, 10, (rows * pitch + 64,), generator=torch.Generator().manual_seed(15)).to(dtype)
    dev = flat.to(DEV)
    view = lambda t: torch.as_strided(t, (rows, n_out), (pitch, 1), offset)
    which, offs = [1, 0], [0, rows - rows // 3, rows]
    SL.surelock_gemm_adapters(x.to(DEV), SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV)), _i32(which), _i32(offs), view(dev))
    want, _ = _want(x, view(flat), a, b, scale, [24] * 2, which, offs)
    assert np.array_equal(view(dev).cpu().double().numpy(), torch.from_numpy(want).to(dtype).double().numpy())
    view(dev).copy_(view(flat))
    assert torch.equal(dev.cpu(), flat)
