"""Sampling from logits with given random numbers, against the definition in 64 bits with a sort.

Tokens and lengths of the prefix are whole numbers and have to be equal: the kernels' sums are off by some 2^-50 of themselves, so a
row differs only where u or a border falls that close to a running sum; the draws here are fixed, and none does.  conf is an
fp32 number of a quotient in 64 bits: 2^-24 of it for its rounding and, where a temperature other than 1 makes fp32 rows sum the plain
softmax apart in 32-bit exponentials, 2^-20."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import build as build_mod

DEV = "cuda"
gpu = pytest.mark.gpu
UNDEFINED = (-1, float("nan"), 0)


def choose(x, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, conf, kept) of one row of float64 logits."""
    if not T >= 0 or np.isnan(x).any() or (x == np.inf).any() or not np.isfinite(x).any():
        return UNDEFINED
    order = np.argsort(-x, kind="stable")
    z = x[order] - x.max()
    soft = np.exp(z) / np.exp(z).sum()
    if T == 0:
        return order[0], soft[0], 1
    with np.errstate(over="ignore"):
        w = np.where(z == 0, 1.0, np.exp(z / T)) if np.isfinite(T) else np.where(np.isfinite(z), 1.0, 0.0)
    n = int(np.isfinite(z).sum())
    w = w[:n]
    if k > 0:
        n = min(n, k)
    cum = np.cumsum(w)
    if p < 1:
        n = min(n, int((cum < p * cum[n - 1]).sum()) + 1)
    if m > 0:
        n = min(n, int((w >= min(m, 1.0)).sum()))
    u = min(max(u, 0.0), float(np.float32(0.99999994))) if u == u else 0.0
    j = min(int((cum <= u * cum[n - 1]).sum()), n - 1)
    return order[j], soft[j], n


def _f32(x):
    return torch.tensor(x, dtype=torch.float32, device=DEV)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _run(logits, u, sampling=None, set_of_row=None, n=None):
    M = logits.shape[0]
    token, conf, kept, status = _i32([-9] * M), _f32([-9] * M), _i32([-9] * M), _i32([0])
    SL.surelock_sample(logits, sampling or SL.Sampling(), _f32(u) if not torch.is_tensor(u) else u, _i32([M if n is None else n]), token, conf, kept, set_of_row, status)
    return token.tolist(), conf.cpu().numpy(), kept.tolist(), status.item()


def _check(logits, u, T=None, k=None, p=None, m=None):
    """One setting for all rows where scalars are given, one per row where lists are."""
    M = logits.shape[0]
    many = isinstance(T, list)
    f32 = lambda v: None if v is None else _f32(v if isinstance(v, list) else [v])
    tokens, conf, kept, status = _run(logits, u, SL.Sampling(f32(T), None if k is None else _i32(k if isinstance(k, list) else [k]), f32(p), f32(m)))
    x = logits.cpu().double().numpy()
    single = lambda v, r, d: d if v is None else float(np.float32(v[r] if isinstance(v, list) else v))
    for r in range(M):
        want = choose(x[r], float(np.float32(u[r])), single(T, r, 1.0), int(single(k, r, 0)), single(p, r, 1.0), single(m, r, 0.0))
        assert (tokens[r], kept[r]) == (want[0], want[2]), (r, tokens[r], kept[r], want)
        assert abs(conf[r] - want[1]) <= 2.0 ** -19 * want[1] or (math.isnan(conf[r]) and math.isnan(want[1])), (r, conf[r], want)
    assert status == 0


def _logits(M, V, dtype, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(M, V, generator=g) * spread
    r = torch.arange(M)
    x[r, torch.randint(0, V, (M,), generator=g)] += 12.0 * (r % 4 == 1)
    if V > 8:
        x[(torch.rand(M, V, generator=g) < 0.4) & (r % 5 == 2)[:, None]] = -math.inf
    return x.to(dtype).to(DEV), torch.rand(M, generator=g).tolist()


# ---- refusals, without a GPU ------------------------------------------------------------------------------------------
def test_refusals_on_the_host():
    build_mod.build()
    L = SL.lib()
    s = lambda n=1: ctypes.byref(SL._Sampling(None, None, None, None, n))
    good = [0x100, 1000, s(), None, 0x200, 0x300, 5, 1000, SL.SL_BF16, 0x400, 0x500, 0x600, None, None]
    for at, value, rc in [(0, None, -1), (1, 999, -1), (2, None, -1), (2, s(0), -1), (2, s(4), -1), (4, None, -1), (5, None, -1), (6, -1, -1), (7, 0, -1), (8, SL.SL_E4M3, -1),
                          (9, None, -1), (0, 0x101, -5), (6, 0, 0)]:
        bad = list(good)
        bad[at] = value
        assert L.surelock_sample(*bad) == rc, (at, value)
    big = list(good)
    big[1] = big[7] = 1 << 20
    assert L.surelock_sample(*big) == -5


# ---- on the GPU -------------------------------------------------------------------------------------------------------
SETTINGS = [dict(), dict(T=0.7), dict(T=0.0), dict(k=1), dict(T=1.3, k=50), dict(p=0.9), dict(p=0.999, T=1.5), dict(m=0.05), dict(T=0.8, k=200, p=0.95, m=0.02), dict(p=0.0), dict(m=1.0)]


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,V", [(1, 126464), (3, 1), (5, 2), (40, 7), (9, 1000), (33, 32003), (70, 16384), (160, 32003), (350, 4099), (2, 200001), (1, 1048000)])
def test_rows(dtype, M, V):
    """One row (a cluster's work) and many, odd vocabularies, confident rows, rows with forbidden tokens."""
    logits, u = _logits(M, V, dtype, M + V)
    for s in SETTINGS if M * V < 500000 else SETTINGS[4::2]:
        _check(logits, u, **s)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_settings_of_their_own(dtype):
    M = 64
    logits, u = _logits(M, 5003, dtype, 1)
    g = np.random.default_rng(2)
    T = [float(t) for t in g.choice([0.0, 0.3, 1.0, 2.0, 1e-30, 1e30, math.inf], M)]
    _check(logits, u, T, g.choice([0, -3, 1, 5, 700, 5003, 99999], M).tolist(), g.choice([1.0, 0.5, 0.99, 2.0, 0.0, -1.0, 1e-9], M).tolist(),
           g.choice([0.0, 0.1, 1.0, 7.0, -2.0, 1e-6], M).tolist())


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("ways", [1, 500])
def test_special_rows(dtype, ways):
    """ways: rows for one CTA each (500) or for clusters of them."""
    V, inf, nan = 20000, math.inf, math.nan
    x = torch.randn(14, V, generator=torch.Generator().manual_seed(3)) * 2
    x[0] = 0.0                                                     # all equal
    x[1] = -7.25
    x[2] = -inf
    x[2, 777] = -3.0                                               # one token left
    x[3] = -inf                                                    # none
    x[4, 12345] = nan
    x[5, 0] = inf
    x[6, ::2], x[6, 1::2] = 0.0, -0.0                              # zeros of either sign are equal
    x[7] = x[7] * 1e-30                                            # tiny, both signs, and zeros
    x[7, 5:900] = -0.0
    x[8, :5] = torch.tensor([3e38, 2.9e38, -3e38, 1e5, 3e38])
    x[9] = torch.linspace(-1e-38, 1e-38, V)                        # subnormal
    x[10, 100:] = -1e30
    x[11, -1] = 30.0                                               # the last token
    x[12] = x[12].sort().values                                    # ascending
    x[13] = -1e4 + x[13]                                           # far from zero
    x = x.to(dtype)
    pick = list(range(14)) * (1 if ways == 1 else ways // 14)
    g = torch.Generator().manual_seed(4)
    u = torch.rand(len(pick), generator=g).tolist()
    for s in (dict(), dict(T=0.5, k=40), dict(p=0.9), dict(m=0.3), dict(T=0.0), dict(k=15000, p=0.99999)):
        if ways == 1:
            for r in pick:
                _check(x[r:r + 1].to(DEV), [u[r]], **s)
        else:
            _check(x[pick].to(DEV), u, **s)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_numbers_at_the_ends(dtype):
    logits, _ = _logits(8, 3000, dtype, 7)
    _check(logits, [0.0, 0.9999999, 1.0, 2.0, -1.0, math.nan, 1e-30, 0.5])
    for T, ok in ((-1.0, False), (math.nan, False)):
        tokens, conf, kept, status = _run(logits, [0.5] * 8, SL.Sampling(_f32([T])))
        assert tokens == [-1] * 8 and np.isnan(conf).all() and kept == [0] * 8 and status == 0
    _check(logits, [0.3] * 8, T=1.0, p=math.nan, m=math.nan)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_frequencies(dtype):
    """u over a fine grid: every token is drawn as often as its probability says, to one draw."""
    n, V = 4000, 50
    row = (torch.randn(V, generator=torch.Generator().manual_seed(8)) * 1.5).to(dtype)
    tokens, _, _, _ = _run(row.repeat(n, 1).to(DEV), ((np.arange(n) + 0.5) / n).tolist(), SL.Sampling(_f32([1.7])))
    z = row.double().numpy() / float(np.float32(1.7))
    p = np.exp(z - z.max())
    assert np.all(np.abs(np.bincount(tokens, minlength=V) - n * p / p.sum()) <= 1 + 1e-3)


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("offset,stride", [(0, 5001), (1, 5003), (3, 5008), (7, 5017)])
def test_rows_anywhere(dtype, offset, stride):
    """Rows that begin off 16 bytes, between other numbers; only the first n rows are drawn."""
    V, M = 5000, 6
    buf = torch.full((M * stride + 64,), float("nan")).to(dtype)
    x, u = _logits(M, V, dtype, 11)
    view = torch.as_strided(buf, (M, V), (stride, 1), offset)
    view.copy_(x.cpu())
    dev = torch.as_strided(buf.to(DEV), (M, V), (stride, 1), offset)
    _check(dev, u, k=300, p=0.9)
    tokens, _, kept, _ = _run(dev, u, n=4)
    assert tokens[4:] == [-9, -9] and kept[4:] == [-9, -9] and tokens[:4] == _run(dev, u)[0][:4]


@gpu
def test_sets_by_row():
    logits, u = _logits(6, 900, torch.bfloat16, 12)
    s = SL.Sampling(_f32([0.0, 1.0, 0.5]), _i32([0, 3, 0]))
    tokens, conf, kept, status = _run(logits, u, s, _i32([2, 0, 1, 1, 3, -1]))
    x = logits.cpu().double().numpy()
    for r, (T, k) in enumerate([(0.5, 0), (0.0, 0), (1.0, 3), (1.0, 3)]):
        assert (tokens[r], kept[r]) == choose(x[r], float(np.float32(u[r])), T, k)[::2]
    assert tokens[4:] == [-1, -1] and kept[4:] == [0, 0] and np.isnan(conf[4:]).all() and status == 4


@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_same_from_a_cluster_and_from_one_cta(dtype):
    logits, _ = _logits(1, 60000, dtype, 13)
    u = torch.rand(600, generator=torch.Generator().manual_seed(14)).tolist()
    for s in (SL.Sampling(), SL.Sampling(_f32([0.6]), _i32([900]), _f32([0.97]), _f32([0.001]))):
        many = _run(logits.expand(600, 60000).contiguous(), u, s)
        few = [_run(logits, [v], s) for v in u[:40]]
        assert many[0][:40] == [f[0][0] for f in few] and many[2][:40] == [f[2][0] for f in few]
        assert [float(c) for c in many[1][:40]] == [float(f[1][0]) for f in few] or np.allclose(many[1][:40], [f[1][0] for f in few], rtol=2.0 ** -22, atol=0)


@gpu
def test_replayed_and_on_several_streams():
    M, V = 20, 30000
    logits, u = _logits(M, V, torch.bfloat16, 15)
    ud, n, tok, kept = _f32(u), _i32([M]), _i32([0] * M), _i32([0] * M)
    s = SL.Sampling(_f32([0.9]), _i32([100]))
    SL.surelock_sample(logits, s, ud, n, tok, None, kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        SL.surelock_sample(logits, s, ud, n, tok, None, kept)
    x = logits.cpu().double().numpy()
    for seed in range(3):
        v = torch.rand(M, generator=torch.Generator().manual_seed(seed))
        ud.copy_(v)
        graph.replay()
        assert tok.tolist() == [choose(x[r], float(v[r]), float(np.float32(0.9)), 100)[0] for r in range(M)]
    want = tok.tolist()
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [_i32([0] * M) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, o in zip(streams, outs):
            with torch.cuda.stream(st):
                SL.surelock_sample(logits, s, ud, n, o)
    torch.cuda.synchronize()
    assert all(o.tolist() == want for o in outs)
