"""Frequency scalings at factors that do not lengthen a context and at contexts shorter than the slowest turns."""
import numpy as np
import pytest

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import build as build_mod


@pytest.mark.parametrize("factor", [0.25, 0.5, 1.0, 1.0 + 2.0 ** -40, 8.0])
def test_yarn_scale(factor):
    """0.1 ln f + 1, but never below 1; one that is given is taken as it is."""
    build_mod.build()
    get = lambda **o: SL.surelock_rope_frequencies(64, 10000.0, "yarn", factor=factor, original_len=4096.0, **o)[1]
    assert get() == np.float32(max(1.0, 0.1 * np.log(factor) + 1.0)) and get(attn_scale=0.75) == 0.75


@pytest.mark.parametrize("length,fast,slow", [(100.0, 32.0, 1.0), (1e9, 32.0, 1.0), (5.0, 4.0, 1.0), (3.0, 9.0, 8.9)])
def test_yarn_borders_stay_within_the_head(length, fast, slow):
    build_mod.build()
    D, theta, f = 64, 10000.0, 4.0
    pair = lambda turns: D * np.log(length / (turns * 2 * np.pi)) / (2 * np.log(theta))
    low, high = max(np.floor(pair(fast)), 0.0), min(np.ceil(pair(slow)), D - 1.0)
    i, w = np.arange(D // 2), theta ** (-np.arange(0, D, 2) / D)
    ramp = np.clip((i - low) / (high - low), 0, 1) if high > low else (i > low).astype(float)
    got = SL.surelock_rope_frequencies(D, theta, "yarn", factor=f, original_len=length, fast=fast, slow=slow)[0].numpy()
    assert np.all(np.abs(got - (w / f * ramp + w * (1 - ramp))) <= 1e-13 * w)
