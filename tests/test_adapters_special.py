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
