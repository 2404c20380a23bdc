"""Adapters beside other kernels that take tensor memory, and numbers at the ends of the types."""
import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL

from . import test_gemm_adapters as ad
from . import test_gemm_quantized as gq
from .test_gemm_adapters import DEV, _i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rank,rows", [(64, 3200), (128, 700)])
def test_followed_by_kernels_that_take_tensor_memory(rank, rows):
    """Products of few rows right behind the adapters of many, launched while those end: the same results as one at a time."""
    a, b, scale = ad._make(2, rank, 512, 256, 21)
    pool = SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV))
    g = torch.Generator().manual_seed(21)
    x = torch.randn(rows, 512, generator=g).to(torch.bfloat16).to(DEV)
    c0 = torch.randn(rows, 256, generator=g).to(DEV)
    which, offs = _i32([0, 1]), _i32([0, rows // 3, rows])
    W, _ = gq._weights(256, 512, 64, True, torch.bfloat16, seed=22)
    dense = torch.randn(256, 512, generator=g).to(torch.bfloat16).to(DEV)
    some, n, status = x[:40].contiguous(), _i32([40]), _i32([0])
    c, few, plain = c0.clone(), torch.zeros(40, 256, dtype=torch.bfloat16, device=DEV), torch.zeros(40, 256, dtype=torch.bfloat16, device=DEV)
    calls = [lambda: SL.surelock_gemm_adapters(x, pool, which, offs, c, status), lambda: SL.surelock_gemm_quantized(some, W, few, n, dev_status=status),
             lambda: SL.surelock_gemm_adapters(x, pool, which, offs, c, status), lambda: SL.surelock_gemm(some, dense, plain, n)]
    for f in calls:
        f()
        torch.cuda.synchronize()
    want = [t.clone() for t in (c, few, plain)]
    for _ in range(20):
        c.copy_(c0)
        few.zero_(), plain.zero_()
        for f in calls:
            f()
    torch.cuda.synchronize()
    assert all(torch.equal(t, w) for t, w in zip((c, few, plain), want)) and status.item() == 0


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cap", [(1, 1), (8, 8), (9, 9), (40, 40), (300, 4000)])
def test_t_keeps_24_bits(dtype, rows, cap):
    """t of 21 bits in three places that two bf16 numbers do not hold; the second product cancels all but the last of them, exactly."""
    a, b = torch.zeros(1, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 40, 16, dtype=torch.bfloat16)
    a[0, 0, :3], a[0, 1, :2] = torch.tensor([1024.0, 32.0, 1.0]), torch.tensor([1024.0, 32.0])
    b[0, :, 0], b[0, :, 1] = 1.0, -1.0
    x = torch.zeros(cap, 64, dtype=torch.bfloat16)
    x[:, :3] = torch.tensor([1024.0, 32.0, 1.0])               # t = 2^20 + 2^10 + 1 and 2^20 + 2^10
    x[::2, 2] = -3.0
    c = torch.zeros(cap, 40, dtype=dtype, device=DEV)
    SL.surelock_gemm_adapters(x.to(DEV), SL.Adapters(a.to(DEV), b.to(DEV), torch.ones(1, device=DEV)), _i32([0]), _i32([0, rows]), c)
    want = torch.zeros(cap, 40)
    want[:rows] = x[:rows, 2:3].float()
    assert torch.equal(c.cpu().float(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rank,rows,cap", [(16, 1, 1), (64, 7, 7), (24, 13, 13), (128, 40, 40), (16, 300, 3100), (72, 300, 700), (128, 200, 400)])
def test_infinite_weights(dtype, rank, rows, cap):
    """Infinities in b, where t is a whole number that one bf16 number holds, one that takes two, and none (zero): infinity or NaN as the
    definition has it, and finite results beside them exact."""
    g = torch.Generator().manual_seed(rank)
    a, b, scale = ad._make(1, rank, 128, 80, 24, exact=True)
    scale[0] = -2.0
    x = torch.randint(-2, 3, (cap, 128), generator=g).to(torch.bfloat16)
    x[:, 0], a[0, :, 0] = 64.0, torch.tensor([256.0, 0.0, -256.0, 128.0] * rank)[:rank].to(torch.bfloat16)
    a[0, 4] = 0.0                                              # this t is zero
    for f, j, v in [(3, 0, "inf"), (5, 1, "-inf"), (9, 2, "inf"), (9, 3, "inf"), (20, 4, "inf"), (33, 7, "-inf"), (64, rank - 1, "inf"), (79, 0, "nan"), (78, 6, "-inf")]:
        b[0, f, j] = float(v)
    c0 = torch.randint(-9, 10, (cap, 80), generator=g).to(dtype)
    c = c0.to(DEV)
    SL.surelock_gemm_adapters(x.to(DEV), SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV)), _i32([0]), _i32([0, rows]), c)
    with np.errstate(invalid="ignore"):
        t = x[:rows].double().numpy() @ a[0].double().numpy().T
        want = c0.double().numpy()
        want[:rows] += (scale[0].item() * t[:, None, :] * b[0].double().numpy()[None]).sum(2)
        size = np.abs(2 * t[:, None, :] * b[0].double().numpy()[None]).sum(2)
    assert size[np.isfinite(size)].max() < 2 ** (21 if rows < 9 else 22) and np.isinf(want).any() and np.isnan(want).any()     # 3 and 2 bits to spare
    assert np.array_equal(c.cpu().double().numpy(), torch.from_numpy(want).to(dtype).double().numpy(), equal_nan=True)


@pytest.mark.parametrize("rows,cap", [(2, 2), (12, 12), (300, 3100)])
def test_t_next_to_the_end_of_its_type(rows, cap):
    """t = 2^128 - 2^116: an fp32 number that no bf16 number is near without being infinite."""
    a, b = torch.zeros(1, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 24, 16, dtype=torch.bfloat16)
    a[0, 0, :12] = 2.0 ** 100
    b[0, :, 0] = 2.0 ** -100
    x = torch.zeros(cap, 64, dtype=torch.bfloat16)
    x[:, :12] = torch.exp2(torch.arange(27, 15, -1).float())
    c = torch.zeros(cap, 24, device=DEV)
    SL.surelock_gemm_adapters(x.to(DEV), SL.Adapters(a.to(DEV), b.to(DEV), torch.tensor([-1.0], device=DEV)), _i32([0]), _i32([0, rows]), c)
    assert bool((c[:rows] == -(2.0 ** 28 - 2.0 ** 16)).all()) and not bool(c[rows:].any())


def test_ranks_above_64_are_summed_as_those_below():
    """t = A x is accumulated in the same four places whatever the rank: b a unit matrix brings it out, and the first 64 ranks of 128 are, bit for
    bit, those of an adapter that has only them.  Rows enough that one CTA takes a tile's whole K."""
    rows, K = 3000 * 128, 512
    g = torch.Generator(device=DEV).manual_seed(26)
    x = torch.randn(rows, K, device=DEV, generator=g).to(torch.bfloat16)
    a = torch.randn(1, 128, K, device=DEV, generator=g).to(torch.bfloat16)
    out = []
    for rank in (64, 128):
        c = torch.zeros(rows, rank, device=DEV)
        unit = torch.eye(rank, device=DEV).to(torch.bfloat16)[None].contiguous()
        SL.surelock_gemm_adapters(x, SL.Adapters(a[:, :rank].contiguous(), unit, torch.ones(1, device=DEV)), _i32([0]), _i32([0, rows]), c)
        out.append(c[:, :64])
    assert torch.equal(*out) and out[0].any()


@pytest.mark.parametrize("offs", [[0] + [1] * 39 + [7], [0] + [2] * 33 + [1] * 7, [0, 1] + [2] * 99 + [-4]])
def test_bad_offsets_behind_the_last_row_are_reported(offs):
    """Every row has its sequence already; the offsets of the many behind them are looked at all the same."""
    a, b, scale = ad._make(2, 16, 64, 32, 27)
    M = max(offs[:2] + offs[2:3])
    x, c0, status = torch.randn(M, 64).to(torch.bfloat16).to(DEV), torch.randn(M, 32, device=DEV), _i32([0])
    SL.surelock_gemm_adapters(x, SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV)), _i32([0] * (len(offs) - 1)), _i32(offs), c0, status)
    assert status.item() == 4
    good, status = [min(max(o, 0), M) for o in np.maximum.accumulate(offs).tolist()], _i32([0])
    SL.surelock_gemm_adapters(x, SL.Adapters(a.to(DEV), b.to(DEV), scale.to(DEV)), _i32([0] * (len(offs) - 1)), _i32(good), c0, status)
    assert status.item() == 0
