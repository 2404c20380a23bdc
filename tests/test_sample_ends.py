"""Sampling at the ends of its settings, against the definition in 64 bits."""

import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL

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
