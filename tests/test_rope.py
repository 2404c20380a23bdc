"""Rotary positions against a statement in 64 bits.

Tolerance per element of a pair, from the roundings: the angle's 2^-53 relative to it is that of the statement too (the same product
in 64 bits, off by 2^-52 of itself between the two); sine and cosine in 32 bits are off by at most 2^-22, the two products and the
sum by 2^-24 each of |a| + |b|, times scale; then the result's own rounding, 2^-8 or 2^-24 of it."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import build as build_mod

DEV = "cuda"
gpu = pytest.mark.gpu
STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def rotate(x, pos, freq, interleaved, scale=1.0, sign=1.0):
    """x [M][H][dh] float64; (result, bound on |a| + |b| per element)."""
    D = 2 * len(freq)
    angle = pos.astype(np.float64)[:, None] * freq
    c, s = np.cos(angle)[:, None], sign * np.sin(angle)[:, None]
    y, size = x.copy(), np.zeros_like(x)
    at = (slice(0, D, 2), slice(1, D, 2)) if interleaved else (slice(0, D // 2), slice(D // 2, D))
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]], y[..., at[1]] = scale * (a * c - b * s), scale * (b * c + a * s)
    size[..., at[0]] = size[..., at[1]] = scale * (np.abs(a) + np.abs(b))
    return y, size


def _check(got, x, pos, freq, interleaved, dtype, scale=1.0, sign=1.0):
    want, size = rotate(x.cpu().double().numpy(), pos, freq, interleaved, scale, sign)
    far = 2.0 ** -52 * np.abs(pos.astype(np.float64)).max(initial=0) * np.abs(freq).max()
    tol = (2.0 ** -21 + far) * size + STEP[dtype] * np.abs(want)
    assert np.all(np.abs(got.cpu().double().numpy() - want) <= tol)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _rope(rot, theta=10000.0, interleaved=False, scale=1.0):
    freq = theta ** (-np.arange(0, rot, 2) / rot)
    return SL.Rope(torch.tensor(freq, device=DEV), interleaved, scale), freq


# ---- refusals and frequencies, without a GPU ----------------------------------------------------------------------------
def test_refusals_on_the_host():
    build_mod.build()
    L = SL.lib()
    cfg = lambda **o: ctypes.byref(SL._RopeCfg(**{**dict(freq=0x1000, rotary_dim=64, interleaved=0, scale=1.0), **o}))
    good = [cfg(), 0x100, 512, 4, 0x200, 256, 2, 128, 0x300, 0, 0x400, 5, 0x500, 512, 0x600, 256, SL.SL_BF16, 0, None, None]
    for at, value, rc in [(0, None, -1), (0, cfg(freq=None), -1), (0, cfg(rotary_dim=0), -1), (0, cfg(rotary_dim=63), -1), (0, cfg(rotary_dim=130), -1), (1, None, -1),
                          (2, 511, -1), (3, 0, -1), (5, 255, -1), (6, 0, -1), (7, 0, -1), (8, None, -1), (9, -1, -1), (10, None, -1), (11, -1, -1), (12, None, -1),
                          (13, 100, -1), (14, None, -1), (15, 1, -1), (16, SL.SL_INT8, -1), (1, 0x101, -5), (0, cfg(freq=0x1004), -5), (7, 5000, -1), (11, 0, 0)]:
        bad = list(good)
        bad[at] = value
        assert L.surelock_rope(*bad) == rc, (at, value)
    bad = list(good)
    bad[12], bad[13] = bad[1], 1024                               # in place with another stride
    assert L.surelock_rope(*bad) == -1


@pytest.mark.parametrize("args", [dict(rotary_dim=0, theta=1e4), dict(rotary_dim=7, theta=1e4), dict(rotary_dim=8, theta=1.0), dict(rotary_dim=8, theta=float("nan")),
                                  dict(rotary_dim=8, theta=1e4, scaling="linear", factor=0.0), dict(rotary_dim=2, theta=1e4, scaling="ntk", factor=2.0),
                                  dict(rotary_dim=8, theta=1e4, scaling="yarn", factor=2.0), dict(rotary_dim=8, theta=1e4, scaling="bands", factor=2.0, original_len=9.0, fast=1.0),
                                  dict(rotary_dim=8, theta=1e4, scaling="other")])
def test_bad_frequencies_are_refused(args):
    build_mod.build()
    with pytest.raises(SL.SurelockError):
        SL.surelock_rope_frequencies(**args)


def test_frequencies():
    build_mod.build()
    D, theta, f, L = 128, 10000.0, 8.0, 4096.0
    w = theta ** (-np.arange(0, D, 2) / D)
    get = lambda **o: (lambda r: (r[0].numpy(), r[1]))(SL.surelock_rope_frequencies(D, theta, **o))
    near = lambda a, b: np.all(np.abs(a - b) <= 1e-13 * b)
    assert near(get()[0], w) and get()[1] == 1.0
    assert near(get(scaling="linear", factor=f)[0], w / f)
    ntk = get(scaling="ntk", factor=f)[0]
    assert near(ntk, (theta * f ** (D / (D - 2))) ** (-np.arange(0, D, 2) / D))
    assert abs(ntk[-1] * f / w[-1] - 1) < 1e-12                    # the slowest pair is slowed by the factor, the fastest not at all
    yarn, m = get(scaling="yarn", factor=f, original_len=L)
    turns = L * w / (2 * math.pi)
    assert near(yarn[turns > 40], w[turns > 40]) and near(yarn[turns < 0.9], w[turns < 0.9] / f) and abs(m - (0.1 * math.log(f) + 1)) < 1e-6
    i = np.arange(D // 2)
    low, high = (math.floor(D * math.log(L / (32 * 2 * math.pi)) / (2 * math.log(theta))), math.ceil(D * math.log(L / (2 * math.pi)) / (2 * math.log(theta))))
    ramp = np.clip((i - low) / (high - low), 0, 1)
    assert near(yarn, w / f * ramp + w * (1 - ramp)) and get(scaling="yarn", factor=f, original_len=L, attn_scale=1.5)[1] == 1.5
    bands = get(scaling="bands", factor=f, original_len=L, fast=4.0, slow=1.0)[0]
    keep = np.clip((turns - 1) / 3, 0, 1)
    assert near(bands, w / f * (1 - keep) + w * keep)


# ---- on the GPU -------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("M,H,Hkv,dh,rot", [(1, 1, 1, 64, 64), (3, 4, 2, 128, 128), (37, 7, 1, 96, 32), (5, 3, 3, 80, 20), (9, 2, 1, 6, 2), (1000, 12, 4, 128, 64),
                                            (2500, 8, 8, 64, 64), (700, 5, 5, 256, 256), (64, 40, 8, 576, 576), (3000, 2, 1, 20, 10)])
def test_rows(dtype, interleaved, M, H, Hkv, dh, rot):
    """Whole and part heads, odd sizes that leave no 16-byte accesses, one row and many; rows behind n_active stay."""
    g = torch.Generator().manual_seed(M + dh)
    rope, freq = _rope(rot, interleaved=interleaved, scale=1.25)
    q, k = (torch.randn(M + 2, h, dh, generator=g).to(dtype).to(DEV) for h in (H, Hkv))
    pos = torch.randint(0, 100000, (M + 2,), generator=g).to(torch.int32)
    qo, ko, status = torch.full_like(q, 7), torch.full_like(k, 7), _i32([0])
    SL.surelock_rope(rope, q, k, pos.to(DEV), _i32([M]), q_out=qo, k_out=ko, dev_status=status)
    for x, y in ((q, qo), (k, ko)):
        _check(y[:M], x[:M], pos[:M].numpy(), freq, interleaved, dtype, 1.25)
        assert torch.equal(y[:M, :, rot:], x[:M, :, rot:]) and bool((y[M:] == 7).all())
    q2, k2 = q.clone(), k.clone()
    SL.surelock_rope(rope, q2, k2, pos.to(DEV), _i32([M]))        # in place: the same
    assert torch.equal(q2[:M], qo[:M]) and torch.equal(k2[:M], ko[:M]) and torch.equal(q2[M:], q[M:])
    q3 = q.clone()
    SL.surelock_rope(rope, q3, None, pos.to(DEV), _i32([M]))      # q alone
    assert torch.equal(q3, q2) and status.item() == 0


@gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(interleaved):
    pos = np.array([0, 1, 2, 8191, 131071, 10 ** 6, 16777217, 10 ** 9 + 7, 2 ** 31 - 1], dtype=np.int64)
    rope, freq = _rope(128, 500000.0, interleaved)
    x = torch.randn(len(pos), 3, 128, generator=torch.Generator().manual_seed(1)).to(DEV)
    y = torch.empty_like(x)
    SL.surelock_rope(rope, x, None, _i32(pos.tolist()), _i32([len(pos)]), q_out=y)
    _check(y, x, pos, freq, interleaved, torch.float32)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_parts_of_wider_rows_and_flat_positions(dtype):
    """q and k as parts of one projection's rows, positions as a step's flat ones, and the inverse."""
    M, H, Hkv, dh, N = 50, 6, 2, 64, 90
    g = torch.Generator().manual_seed(4)
    wide = torch.randn(M, H + 2 * Hkv, dh, generator=g).to(dtype).to(DEV)
    keep = wide.clone()
    idx = torch.randint(0, 7 * N, (M,), generator=g).to(torch.int32)
    rope, freq = _rope(64)
    SL.surelock_rope(rope, wide[:, :H], wide[:, H:H + Hkv], idx.to(DEV), _i32([M]), N=N)
    pos = (idx % N).numpy()
    _check(wide[:, :H + Hkv], keep[:, :H + Hkv], pos, freq, False, dtype)
    assert torch.equal(wide[:, H + Hkv:], keep[:, H + Hkv:])
    turned = wide.clone()
    SL.surelock_rope(rope, wide[:, :H], wide[:, H:H + Hkv], idx.to(DEV), _i32([M]), N=N, transposed=True)
    _check(wide[:, :H + Hkv], turned[:, :H + Hkv], pos, freq, False, dtype, sign=-1.0)


@gpu
def test_a_step_of_the_context_rotates_alike():
    """On the step's own conventions (half layout, whole head, position = flat index mod N) a rotation keeps q.k of two rows a
    function of their distance."""
    rope, _ = _rope(128)
    g = torch.Generator().manual_seed(5)
    q, k = (torch.randn(1, 1, 128, generator=g).to(DEV) for _ in range(2))
    dots = []
    for a, b in [(5, 2), (1005, 1002), (300003, 300000)]:
        qa, kb = q.clone(), k.clone()
        SL.surelock_rope(rope, qa, None, _i32([a]), _i32([1]))
        SL.surelock_rope(rope, kb, None, _i32([b]), _i32([1]))
        dots.append((qa.double() * kb.double()).sum().item())
    size = (q.abs() * k.abs()).sum().item()
    assert max(dots) - min(dots) <= 2 * 2.0 ** -19 * 2 * size


@gpu
def test_bad_positions_leave_rows_and_special_values_stay_in_their_pairs():
    rope, freq = _rope(64)
    x = torch.randn(4, 2, 64, generator=torch.Generator().manual_seed(6)).to(DEV)
    x[2, 1, 3], x[3, 0, 40] = float("nan"), float("inf")
    y, status = torch.full_like(x, 3.0), _i32([0])
    SL.surelock_rope(rope, x, None, _i32([5, -1, 7, 8]), _i32([4]), q_out=y, dev_status=status)
    assert status.item() == 4 and bool((y[1] == 3.0).all())
    bad = ~torch.isfinite(y)
    want = torch.zeros_like(bad)
    want[2, 1, 3] = want[2, 1, 35] = want[3, 0, 8] = want[3, 0, 40] = True
    assert torch.equal(bad, want)


@gpu
def test_gradient():
    """The transposed call is the gradient: <R x, y> = <x, R' y>, and differences of a linear map are exact but for roundings."""
    rope, freq = _rope(32, interleaved=True, scale=0.75)
    g = torch.Generator().manual_seed(8)
    x, y = (torch.randn(20, 3, 48, generator=g).to(DEV) for _ in range(2))
    pos = torch.randint(0, 5000, (20,), generator=g).to(torch.int32).to(DEV)
    rx, ry = torch.empty_like(x), torch.empty_like(x)
    SL.surelock_rope(rope, x, None, pos, _i32([20]), q_out=rx)
    SL.surelock_rope(rope, y, None, pos, _i32([20]), q_out=ry, transposed=True)
    a, b = (rx.double() * y.double()).sum().item(), (x.double() * ry.double()).sum().item()
    assert abs(a - b) <= 2 * 2.0 ** -20 * 2 * (x.abs() * y.abs()).double().sum().item() + 2 * 2.0 ** -20 * x.abs().double().sum().item() * 4


@gpu
def test_replayed_with_other_positions_and_counts():
    M = 64
    rope, freq = _rope(128)
    x = torch.randn(M, 4, 128, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).to(DEV)
    y, pos, n = torch.zeros_like(x), _i32([0] * M), _i32([M])
    SL.surelock_rope(rope, x, None, pos, n, q_out=y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        SL.surelock_rope(rope, x, None, pos, n, q_out=y)
    for seed, m in enumerate([64, 1, 0, 33]):
        p = torch.randint(0, 9000, (M,), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        pos.copy_(p)
        n.fill_(m)
        y.zero_()
        graph.replay()
        _check(y[:m], x[:m], p[:m].numpy(), freq, False, torch.bfloat16)
        assert not y[m:].any()
