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
