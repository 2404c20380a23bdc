"""Sampling at the ends of its settings, against the definition in 64 bits."""

import ctypes

import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import build as build_mod

from .test_sample import DEV, _check, _run

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,V,far", [(3, 126464, False), (3, 126464, True), (40, 3001, False), (200, 20000, True)])
def test_small_min_p(dtype, M, V, far):
    """min-p far below the units of the sums (2^-54 of the largest weight), in both methods for bf16 rows (far: a value outside the window).  The
    length is a whole number: a token is kept if its weight is at least min-p, however small both are."""
    g = torch.Generator().manual_seed(V + M)
    x = torch.randn(M, V, generator=g) * 6
    x[:, 7] = x.max(dim=1).values - 40.0
    if far:
        x[:, 11] = -1e5
    logits, u = x.to(dtype).to(DEV), torch.rand(M, generator=g).tolist()
    for m in (1e-8, 1e-12, 1e-14, 3e-16, 1e-16, 1e-18, 1e-20, 1e-30, 1e-44):
        _check(logits, u, m=m)
    _check(logits, u, T=1.7, k=V - 5, m=1e-19)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,V,far", [(1, 126464, False), (5, 126464, True), (200, 20000, False), (300, 777, True)])
def test_conf_is_a_quotient_in_64_bits(dtype, M, V, far):
    """At any temperature conf is off by its own rounding to fp32 and the sum's errors: exponentials of 2^-47 and V additions of 2^-53 each at most, far
    below it.  A logit's distance from the largest is exact in 64 bits."""
    g = torch.Generator().manual_seed(V + M)
    x = torch.randn(M, V, generator=g) * 2
    if far:
        x[:, 11] = -1e5
    logits, u = x.to(dtype), torch.rand(M, generator=g).tolist()
    for T in (0.7, 1.0, 2.5):
        tokens, conf, _, _ = _run(logits.to(DEV), u, SL.Sampling(torch.tensor([T], device=DEV)))
        z = logits.double().numpy()
        z -= z.max(axis=1, keepdims=True)
        want = np.exp(z[np.arange(M), tokens]) / np.exp(z).sum(axis=1)
        assert np.all(np.abs(conf.astype(np.float64) - want) <= (2.0 ** -24 + 2.0 ** -35) * want)


def test_a_vocabulary_too_large_is_refused_on_the_host():
    build_mod.build()
    sets = ctypes.byref(SL._Sampling(None, None, None, None, 1))
    V = (1 << 20) - 127
    assert SL.lib().surelock_sample(0x100, V, sets, None, 0x200, 0x300, 5, V, SL.SL_BF16, 0x400, 0x500, 0x600, None, None) == -5


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_largest_vocabulary(dtype):
    V = (1 << 20) - 128
    g = torch.Generator().manual_seed(28)
    x = torch.randn(2, V, generator=g)
    x[1] = 0.0                                                 # as many tokens as there are in one bin
    for T, k, p in ((1.0, 0, 1.0), (3.0, V - 1, 0.999)):
        _check(x.to(dtype).to(DEV), [0.999, 0.9999], T=T, k=k, p=p)
