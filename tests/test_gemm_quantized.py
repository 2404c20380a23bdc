"""Products with 4-bit weights against plain statements in 64 bits.

Two kinds of case.  With small whole numbers in A and powers of two as scales every product, group sum and total is exact in
fp32 in any order, so the fp32 epilogue is compared bit for bit: that pins every index.  With random values the bound is
that of the summation: a lane's chain is K / 16 matrix instructions and K / group scaled adds, then at most 64 partial sums
are joined; each step is off by at most 2^-22 of sum |a| |w| (an fp32 addition that may truncate: 2^-23, twice over for the
sum inside the instruction); a bf16 result is off by half a step more, 2^-8 of its value.  silu(x) y: the derivative of
silu is at most 1.1 and |silu(x)| <= |x|, and its exponential is off by 2^-20 of it at most."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import build as build_mod

DEV = "cuda"
gpu = pytest.mark.gpu


def _weights(n, K, group, zeros, scale_t, seed, exact=False):
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 256, (n, K // 2), generator=g, dtype=torch.uint8)
    if exact:
        scales = torch.exp2(torch.randint(-2, 3, (n, K // group), generator=g).float()).to(scale_t)
    else:
        scales = (torch.randn(n, K // group, generator=g) * 0.02).to(scale_t)          # either sign
    z = torch.randint(0, 16, (n, K // group), generator=g, dtype=torch.uint8) if zeros else None
    u = torch.stack([codes & 15, codes >> 4], 2).reshape(n, K).double().numpy()
    w = (u.reshape(n, -1, group) - (z.double().numpy()[..., None] if zeros else 8)) * scales.double().numpy()[..., None]
    return tuple(t.to(DEV) if t is not None else None for t in (codes, scales, z)), w.reshape(n, K)


def _run(A, W, C, M, epilogue, W2=None):
    SL.surelock_gemm_quantized(A, W, C, torch.tensor([M], dtype=torch.int32, device=DEV), epilogue=epilogue, W2=W2)


# ---- refusals, without a GPU ------------------------------------------------------------------------------------------
def test_refusals_on_the_host():
    build_mod.build()
    L = SL.lib()
    W = lambda **o: ctypes.byref(SL._W4(**{**dict(codes=0x1000, scales=0x2000, zeros=None, group=64, scale_dtype=SL.SL_BF16), **o}))
    good = [0x100, W(), None, 0x200, 0x300, 4, 10, 128, 0, 0x1000, None, None]
    cases = [(0, None, -1), (1, None, -1), (3, None, -1), (4, None, -1), (5, -1, -1), (6, 0, -1), (7, 0, -1), (7, 96, -1), (8, 3, -1), (8, -1, -1),
             (1, W(codes=None), -1), (1, W(scales=None), -1), (1, W(group=0), -1), (1, W(scale_dtype=SL.SL_INT8), -1), (1, W(group=16), -5),
             (1, W(codes=0x1008), -5), (0, 0x108, -5), (8, 2, -1), (9, None, -1), (9, 0x1080, -5), (5, 0, 0)]
    for at, value, rc in cases:
        bad = list(good)
        bad[at] = value
        assert L.surelock_gemm_quantized(*bad) == rc, (at, value)
    swiglu = [0x100, W(), W(), 0x200, 0x300, 4, 10, 128, 2, 0x1000, None, None]
    for w2 in (W(group=32), W(scale_dtype=SL.SL_FP32), W(zeros=0x3000), W(codes=None)):
        swiglu[2] = w2
        assert L.surelock_gemm_quantized(*swiglu) == -1


def test_binding_refuses_wrong_shapes():
    A, C = torch.zeros(2, 128, dtype=torch.bfloat16), torch.zeros(2, 5, dtype=torch.bfloat16)
    codes, scales = torch.zeros(5, 64, dtype=torch.uint8), torch.zeros(5, 2)
    n = torch.zeros(1, dtype=torch.int32)
    for a, w, c, e in [(A.float(), (codes, scales, None), C, 0), (A, (codes, scales, None), C, 1), (A, (codes[:, :32].contiguous(), scales, None), C, 0),
                       (A, (codes, scales[:, :1].expand(5, 3), None), C, 0), (A, (codes, scales, scales), C, 0), (A, (codes, scales, None), C[:1], 0)]:
        with pytest.raises(SL.SurelockError):
            SL.surelock_gemm_quantized(a, w, c, n, epilogue=e)


# ---- exact cases ------------------------------------------------------------------------------------------------------
SHAPES = [  # M, n_out, K, group
    (1, 1, 32, 32), (1, 17, 128, 128), (3, 100, 96, 32), (8, 129, 192, 64), (9, 64, 640, 128), (23, 200, 1056, 32), (16, 40, 1344, 64),
    (33, 130, 256, 64), (64, 65, 384, 128), (65, 33, 512, 128), (128, 300, 1280, 64), (130, 48, 4096, 128), (1, 1000, 4096, 128), (5, 37, 12288, 64),
    (40, 72, 13824, 128), (64, 31, 12320, 32), (7, 4096, 4096, 128), (100, 777, 2048, 32),
]


@gpu
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("scale_t", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,n,K,group", SHAPES)
def test_whole_numbers_are_exact(M, n, K, group, zeros, scale_t):
    W, w = _weights(n, K, group, zeros, scale_t, seed=M + n, exact=True)
    g = torch.Generator().manual_seed(K)
    a = torch.randint(-4, 5, (M + 3, K), generator=g)
    a[M:] = 1 << 10                                                   # rows behind the count take no part
    A = a.to(torch.bfloat16).to(DEV)
    C = torch.randint(-8, 9, (M + 3, n), generator=g).float()
    want = C.double().numpy()
    want[:M] += a[:M].double().numpy() @ w.T
    D = C.to(DEV)
    _run(A, W, D, M, 1)
    assert np.array_equal(D.cpu().double().numpy(), want)
    D = torch.full((M + 3, n), 7.0, dtype=torch.bfloat16, device=DEV)
    _run(A, W, D, M, 0)
    want0 = torch.from_numpy(want[:M] - C[:M].double().numpy()).float().to(torch.bfloat16)
    assert torch.equal(D[:M].cpu(), want0) and torch.all(D[M:] == 7.0)


# ---- random cases -----------------------------------------------------------------------------------------------------
def _tol(A, w, K, group):
    return (K / 16 + K / group + 64) * 2.0 ** -22 * (np.abs(A) @ np.abs(w).T)


@gpu
@pytest.mark.parametrize("M,n,K,group,zeros,scale_t,epilogue", [
    (1, 4096, 4096, 128, False, torch.bfloat16, 0), (23, 1000, 4096, 128, True, torch.bfloat16, 2), (128, 515, 2048, 64, True, torch.float32, 1),
    (8, 300, 1024, 32, False, torch.float32, 2), (64, 129, 768, 64, False, torch.bfloat16, 2), (12, 77, 96, 32, True, torch.bfloat16, 2),
    (90, 200, 640, 128, True, torch.float32, 2), (31, 2049, 5120, 128, False, torch.float32, 0), (2, 50, 12288, 64, True, torch.float32, 1)])
def test_random_values(M, n, K, group, zeros, scale_t, epilogue):
    W, w = _weights(n, K, group, zeros, scale_t, seed=1)
    g = torch.Generator().manual_seed(2)
    A = (torch.randn(M, K, generator=g) * torch.exp(torch.randn(M, 1, generator=g))).to(torch.bfloat16)
    a = A.double().numpy()
    x, tx = a @ w.T, _tol(a, w, K, group)
    W2 = None
    if epilogue == 2:
        W2, w2 = _weights(n, K, group, zeros, scale_t, seed=3)
        y, ty = a @ w2.T, _tol(a, w2, K, group)
        s = x / (1 + np.exp(-x))
        want, tol = s * y, 1.1 * tx * (np.abs(y) + ty) + np.abs(s) * (ty + 2.0 ** -20 * np.abs(y))
    else:
        want, tol = x, tx
    if epilogue == 1:
        C = torch.randn(M, n, generator=g)
        want = want + C.double().numpy()
        tol = tol + 2.0 ** -24 * np.abs(want)
        D = C.to(DEV)
    else:
        tol = tol + 2.0 ** -8 * np.abs(want)
        D = torch.empty(M, n, dtype=torch.bfloat16, device=DEV)
    keep = D.clone()
    _run(A.to(DEV), W, D, M, epilogue, W2)
    d = np.abs(D.cpu().double().numpy() - want)
    assert np.all(d <= tol), float((d / tol).max())
    again = keep
    _run(A.to(DEV), W, again, M, epilogue, W2)
    assert torch.equal(again, D)                                      # the same bits again


@gpu
def test_rows_do_not_meet():
    """A row of infinities or NaN leaves the others as they are; large finite values stay finite."""
    W, w = _weights(64, 256, 64, True, torch.bfloat16, seed=5)
    A = torch.randn(12, 256, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    D = torch.empty(12, 64, dtype=torch.bfloat16, device=DEV)
    _run(A.to(DEV), W, D, 12, 0)
    B = A.clone()
    B[3] = float("inf")
    B[10, 7] = float("nan")
    B[5] = A[5] * 2.0 ** 100
    E = torch.empty_like(D)
    _run(B.to(DEV), W, E, 12, 0)
    rest = [r for r in range(12) if r not in (3, 5, 10)]
    assert torch.equal(D[rest], E[rest]) and torch.all(torch.isnan(E[10]))
    assert torch.equal(E[5].float(), D[5].float() * 2.0 ** 100)


@gpu
def test_graph_streams_and_changing_counts():
    M, n, K = 20, 600, 1024
    W, w = _weights(n, K, 128, False, torch.bfloat16, seed=7)
    A = torch.randn(M, K, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to(DEV)
    want = torch.zeros(M, n, dtype=torch.bfloat16, device=DEV)
    _run(A, W, want, M, 0)
    count = torch.tensor([M], dtype=torch.int32, device=DEV)
    out = torch.zeros_like(want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        SL.surelock_gemm_quantized(A, W, out, count)
    for m in (20, 0, 1, 13):
        out.zero_()
        count.fill_(m)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:m], want[:m]) and torch.all(out[m:] == 0)
    streams, outs = [torch.cuda.Stream() for _ in range(3)], [torch.zeros_like(want) for _ in range(3)]
    count.fill_(M)
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o in zip(streams, outs):
            with torch.cuda.stream(s):
                SL.surelock_gemm_quantized(A, W, o, count)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


# ---- what the shapes above leave out --------------------------------------------------------------------------------
def test_outputs_that_cannot_be_written_in_fours_are_refused():
    build_mod.build()
    L = SL.lib()
    w = ctypes.byref(SL._W4(codes=0x1000, scales=0x2000, zeros=None, group=64, scale_dtype=SL.SL_BF16))
    for epilogue, c, rc in [(0, 0x204, -5), (0, 0x202, -5), (2, 0x204, -5), (0, 0x208, 0), (1, 0x204, 0)]:
        assert L.surelock_gemm_quantized(0x100, w, w, c, 0x300, 0, 10, 128, epilogue, 0x1000, None, None) == rc


@gpu
@pytest.mark.parametrize("scale_t", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,n,K,group", [(2, 70, 1344, 64), (19, 130, 640, 128), (32, 64, 416, 32), (20, 4800, 160, 32), (26, 5003, 192, 64), (3, 40, 20480, 128), (37, 33, 18464, 32), (34, 200, 1056, 32), (50, 70, 1344, 64), (127, 257, 1280, 64),
                                         (128, 131, 1152, 128), (129, 40, 160, 32)])
def test_large_zero_points_are_exact(M, n, K, group, scale_t):
    """Zero points over their whole range, 0 ... 127; |sum| <= 1344 x 4 x 127 x 4 < 2^24, so the whole numbers stay exact."""
    (codes, scales, _), _ = _weights(n, K, group, False, scale_t, seed=M, exact=True)
    g = torch.Generator().manual_seed(M)
    z = torch.randint(0, 128, (n, K // group), generator=g, dtype=torch.uint8)
    z[:, 0], z[0] = 127, 0
    c = codes.cpu()
    u = torch.stack([c & 15, c >> 4], 2).reshape(n, -1, group).double().numpy()
    w = ((u - z.double().numpy()[..., None]) * scales.cpu().double().numpy()[..., None]).reshape(n, K)
    a = torch.randint(-4, 5, (M, K), generator=g)
    D = torch.zeros(M, n, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    SL.surelock_gemm_quantized(a.to(torch.bfloat16).to(DEV), (codes, scales, z.to(DEV)), D, torch.tensor([M], dtype=torch.int32, device=DEV),
                               epilogue=1, dev_status=status)
    assert np.array_equal(D.cpu().double().numpy(), a.double().numpy() @ w.T) and status.item() == 0


@gpu
@pytest.mark.parametrize("scale_t", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,n,K,group", [(4, 66, 256, 32), (16, 190, 640, 64), (30, 129, 1152, 128), (18, 2500, 352, 32), (29, 2437, 256, 128), (33, 66, 800, 32), (64, 190, 640, 64), (65, 129, 1152, 128),
                                         (100, 65, 2112, 64), (128, 640, 512, 128), (131, 100, 96, 32)])
def test_swiglu(M, n, K, group, scale_t):
    W, w = _weights(n, K, group, True, scale_t, seed=M)
    W2, w2 = _weights(n, K, group, True, scale_t, seed=M + 1)
    A = torch.randn(M + 1, K, generator=torch.Generator().manual_seed(M)).to(torch.bfloat16)
    a = A[:M].double().numpy()
    x, tx, y, ty = a @ w.T, _tol(a, w, K, group), a @ w2.T, _tol(a, w2, K, group)
    s = x / (1 + np.exp(-x))
    want = s * y
    tol = 1.1 * tx * (np.abs(y) + ty) + np.abs(s) * (ty + 2.0 ** -20 * np.abs(y)) + 2.0 ** -8 * np.abs(want)
    D = torch.full((M + 1, n), 7.0, dtype=torch.bfloat16, device=DEV)
    _run(A.to(DEV), W, D, M, 2, W2)
    d = np.abs(D[:M].cpu().double().numpy() - want)
    assert np.all(d <= tol), float((d / tol).max())
    assert torch.all(D[M:] == 7.0)


@gpu
@pytest.mark.parametrize("M,counts", [(70, (70, 0, 1, 33, 64, 65)), (200, (200, 128, 129, 7))])
def test_many_rows_under_a_graph_with_changing_counts(M, counts):
    """A workspace that holds NaN, counts below the capacity, and a replay beside calls on another stream."""
    n, K = 200, 1056
    W, w = _weights(n, K, 32, True, torch.bfloat16, seed=9)
    A = torch.randn(M, K, generator=torch.Generator().manual_seed(10)).to(torch.bfloat16).to(DEV)
    want = torch.zeros(M, n, dtype=torch.bfloat16, device=DEV)
    _run(A, W, want, M, 0)
    count, full = (torch.tensor([M], dtype=torch.int32, device=DEV) for _ in range(2))
    out, beside = torch.zeros_like(want), torch.zeros_like(want)
    ws = torch.full((SL.surelock_gemm_quantized_workspace_bytes(M, K),), 255, dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        SL.surelock_gemm_quantized(A, W, out, count, workspace=ws, dev_status=status)
    other = torch.cuda.Stream()
    for m in counts:
        out.zero_()
        beside.zero_()
        ws.fill_(255)
        count.fill_(m)
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            SL.surelock_gemm_quantized(A, W, beside, full, dev_status=status)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:m], want[:m]) and torch.all(out[m:] == 0) and torch.equal(beside, want)
    assert status.item() == 0


@gpu
def test_refusals_with_tensors(monkeypatch):
    W, _ = _weights(40, 128, 64, False, torch.bfloat16, seed=11)
    A, C, one = torch.zeros(2, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 40, dtype=torch.bfloat16, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    SL.surelock_gemm_quantized(A[:0], W, C[:0], one)                  # no rows: nothing to do
    wide = torch.zeros(81, dtype=torch.bfloat16, device=DEV)
    for bad in [(A, W, C, one.cpu()), (A, W, C, one.long()), (A, (W[0].cpu(), *W[1:]), C, one), (A, W, wide[1:].reshape(2, 40), one), (A.cpu(), W, C, one)]:
        with pytest.raises(SL.SurelockError):
            SL.surelock_gemm_quantized(*bad)
    with pytest.raises(SL.SurelockError):
        SL.surelock_gemm_quantized(A, W, C, one, workspace=torch.zeros(8, dtype=torch.uint8, device=DEV))
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)       # as if another device were the current one
    with pytest.raises(SL.SurelockError):
        SL.surelock_gemm_quantized(A, W, C, one)


# ---- alignment of scales and of an fp32 output ------------------------------------------------------------------------
def test_elements_off_their_alignment_are_refused():
    """Read or written one at a time, which the device cannot do off an element's alignment.  Without rows: nothing is launched."""
    build_mod.build()
    L = SL.lib()
    w = lambda at, t: ctypes.byref(SL._W4(codes=0x1000, scales=at, zeros=None, group=64, scale_dtype=t))
    call = lambda a, b, c, epilogue: L.surelock_gemm_quantized(0x100, a, b, c, 0x300, 0, 10, 128, epilogue, 0x1000, None, None)
    for t, at, rc in [(SL.SL_BF16, 0x2001, -5), (SL.SL_BF16, 0x2002, 0), (SL.SL_FP32, 0x2002, -5), (SL.SL_FP32, 0x2001, -5), (SL.SL_FP32, 0x2004, 0)]:
        assert call(w(at, t), None, 0x200, 0) == rc
        assert call(w(0x2000, t), w(at, t), 0x200, 2) == rc           # and of the second matrix
    for c, rc in [(0x202, -5), (0x201, -5), (0x204, 0)]:
        assert call(w(0x2000, SL.SL_BF16), None, c, 1) == rc


def test_binding_refuses_other_numbers_of_dimensions():
    A, C = torch.zeros(2, 128, dtype=torch.bfloat16), torch.zeros(2, 5, dtype=torch.bfloat16)
    codes, scales, n = torch.zeros(5, 64, dtype=torch.uint8), torch.zeros(5, 2), torch.zeros(1, dtype=torch.int32)
    for a, w, w2 in [(A, (codes, scales[:, 0], None), None), (A, (codes, scales[None], None), None), (A[0], (codes, scales, None), None),
                     (A[None], (codes, scales, None), None), (A, (codes, scales), None), (A, (codes, scales, None), (codes, scales[0], None))]:
        with pytest.raises(SL.SurelockError):
            SL.surelock_gemm_quantized(a, w, C, n, epilogue=2 if w2 else 0, W2=w2)


# ---- the same on both kernels: up to 16 rows, up to 32 of many features, and more ------------------------------------------
KERNELS = [(13, 600), (20, 4800), (20, 600), (33, 200), (70, 200), (128, 130)]


@gpu
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,n", KERNELS)
def test_counts_replays_and_streams(M, n, group):
    """Workspaces full of NaN (rows behind the count are not rewritten), counts that change between replays of one graph, and calls
    on three streams at once, each with a workspace of its own."""
    K = 1152
    W, _ = _weights(n, K, group, True, torch.bfloat16, seed=9)
    A = torch.randn(M, K, generator=torch.Generator().manual_seed(10)).to(torch.bfloat16).to(DEV)
    want = torch.zeros(M, n, dtype=torch.bfloat16, device=DEV)
    _run(A, W, want, M, 0)
    space = lambda: torch.full((SL.surelock_gemm_quantized_workspace_bytes(M, K),), 255, dtype=torch.uint8, device=DEV)
    count, out, ws, status = torch.tensor([M], dtype=torch.int32, device=DEV), torch.zeros_like(want), space(), torch.zeros(1, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        SL.surelock_gemm_quantized(A, W, out, count, workspace=ws, dev_status=status)
    for m in (M, 0, 1, M - 1, 9, M):
        out.fill_(7.0)
        ws.fill_(255)
        count.fill_(m)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[:m], want[:m]) and torch.all(out[m:] == 7.0)
    streams, outs, spaces = [torch.cuda.Stream() for _ in range(3)], [torch.zeros_like(want) for _ in range(3)], [space() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o, w in zip(streams, outs, spaces):
            with torch.cuda.stream(s):
                SL.surelock_gemm_quantized(A, W, o, count, workspace=w, dev_status=status)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs) and status.item() == 0


@gpu
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,n", KERNELS)
def test_rows_do_not_meet_in_either_kernel(M, n, group):
    K = 640
    W, _ = _weights(n, K, group, True, torch.bfloat16, seed=5)
    A = torch.randn(M, K, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    D, E = (torch.empty(M, n, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    _run(A.to(DEV), W, D, M, 0)
    B = A.clone()
    B[3], B[M - 1, 7], B[5] = float("inf"), float("nan"), A[5] * 2.0 ** 100
    _run(B.to(DEV), W, E, M, 0)
    rest = [r for r in range(M) if r not in (3, 5, M - 1)]
    assert torch.equal(D[rest], E[rest]) and torch.all(torch.isnan(E[M - 1])) and torch.all(torch.isnan(E[3]))
    assert torch.equal(E[5].float(), D[5].float() * 2.0 ** 100)


@gpu
@pytest.mark.parametrize("most", [16, 128])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,n", KERNELS)
def test_rows_with_a_common_mean(M, n, group, most):
    """Where sum (u - z) a is small beside its two shares.  The kernel for few rows subtracts them: its roundings are relative to
    sum |a| (u + z) s (the shares' chains are as long as those of the bound above).  The other takes z off the codes, exactly: to
    sum |a| |u - z| s, and groups of codes at their zero point give an exact 0."""
    K = 1152
    (codes, scales, _), _ = _weights(n, K, group, False, torch.float32, seed=4)
    g = torch.Generator().manual_seed(M)
    z = torch.randint(0, most, (n, K // group), generator=g, dtype=torch.uint8)
    codes, scales = codes.cpu(), scales.cpu()
    z[0] = torch.randint(0, 16, z[0].shape, generator=g, dtype=torch.uint8)
    codes[0] = (z[0] * 17).repeat_interleave(group // 2)              # feature 0: every code its zero point
    u = torch.stack([codes & 15, codes >> 4], 2).reshape(n, -1, group).double().numpy()
    s = scales.double().numpy()[..., None]
    w, both = (((u - z.double().numpy()[..., None]) * s).reshape(n, K), ((u + z.double().numpy()[..., None]) * np.abs(s)).reshape(n, K))
    A = (5 + 0.1 * torch.randn(M, K, generator=g)).to(torch.bfloat16)
    a = A.double().numpy()
    D = torch.zeros(M, n, device=DEV)
    _run(A.to(DEV), (codes.to(DEV), scales.to(DEV), z.to(DEV)), D, M, 1)
    want, few = a @ w.T, M <= 16 or (M <= 32 and n > 128 * 37)
    d, tol = np.abs(D.cpu().double().numpy() - want), _tol(a, both if few else w, K, group) + 2.0 ** -24 * np.abs(want)
    assert np.all(d <= tol), float((d / np.maximum(tol, 1e-30)).max())
    assert few or torch.all(D[:, 0] == 0)


# ---- far ends -----------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("M,n,K,group", [(9, 70, 640, 64), (40, 70, 640, 128), (100, 33, 320, 32)])
@pytest.mark.parametrize("power", [-133, -126, -100, 100, 112])
def test_rows_of_any_magnitude_are_exact(M, n, K, group, power):
    """Whole numbers up to 4 times a power of two, down to subnormal bf16 rows and fp32 results: |sum| < 2^15 quarters, so every
    result is a number of fp32 and the powers only move its exponent."""
    W, w = _weights(n, K, group, True, torch.float32, seed=M, exact=True)
    a = torch.randint(-4, 5, (M, K), generator=torch.Generator().manual_seed(M)).double()
    a[1] = 0
    D = torch.zeros(M, n, device=DEV)
    _run((a * 2.0 ** power).to(torch.bfloat16).to(DEV), W, D, M, 1)
    assert np.array_equal(D.cpu().double().numpy(), (a.numpy() @ w.T) * 2.0 ** power)


@gpu
@pytest.mark.parametrize("M,n,K,group", [(1, 2 ** 31 - 1, 32, 32), (2, 150001, 40960, 128), (33, 150001, 40960, 64)])
def test_codes_beyond_32_bits(M, n, K, group):
    """More than 2^31 bytes of codes, and the most features there can be: the first, the last and some features between."""
    at = [0, 1, 127, 128, n // 2, n // 2 + 5, n - 130, n - 2, n - 1]
    W, w = _weights(len(at), K, group, True, torch.bfloat16, seed=3, exact=True)
    codes = torch.zeros(n, K // 2, dtype=torch.uint8, device=DEV)
    scales = torch.zeros(n, K // group, dtype=torch.bfloat16, device=DEV)
    zeros = torch.zeros(n, K // group, dtype=torch.uint8, device=DEV)
    for i, f in enumerate(at):
        codes[f], scales[f], zeros[f] = W[0][i], W[1][i], W[2][i]
    a = torch.randint(-4, 5, (M, K), generator=torch.Generator().manual_seed(4))
    a[:, 4096:] = 0                                                   # so that the whole numbers stay exact
    D = torch.full((M, n), 7.0, dtype=torch.bfloat16, device=DEV)
    _run(a.to(torch.bfloat16).to(DEV), (codes, scales, zeros), D, M, 0)
    want = torch.from_numpy(a.double().numpy() @ w.T).float().to(torch.bfloat16)
    assert torch.equal(torch.stack([D[:, f] for f in at], 1).cpu(), want)
    D[:, torch.tensor(at, device=DEV)] = 0
    assert not D.any()
    del codes, scales, zeros, D
    torch.cuda.empty_cache()                                          # some 40 GB, which later tests need not find taken
