"""Paged K/V cache: writing (quantised), reading back and attention, against plain statements in 64 bits.

Codes and scales are compared bit for bit.  Tolerance of the attention, per output element, from its roundings: the output
is rounded to bf16 (2^-8 of its value); the weights enter the product with V rounded by half a step of fp16 (2^-11) or, over
a bf16 cache, of bf16 (2^-8), which moves the result by at most that times A = sum p |v| / sum p.  The rest (fp32
accumulation of at most 128 products, a score in fp32, the 2^-22 of exp2, q elements below 2^-14 of their row's largest in
fp16) stays below 2^-12 A for scores up to some hundreds: |s| 2^-22 for the score, 128 x 2^-24 for its sum.  Over an 8-bit
cache a weight w_j = p_j * scale_j is an fp16 number whose row's largest is at least 2^8, so a weight below fp16's normal
numbers is off by at most 2^-25 / 2^8 = 2^-33 of the largest weight W = max_j w_j / sum p: n such weights, times codes of at
most Q, move the result by at most n Q 2^-33 W."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import build as build_mod

DEV = "cuda"
QMAX = {torch.float8_e4m3fn: 448.0, torch.int8: 127.0}
KINDS = [torch.bfloat16, torch.float8_e4m3fn, torch.int8]
E4M3 = np.array([(m / 8.0) * 2.0 ** -6 for m in range(8)] +
                [(1 + m / 8.0) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1])


def quantise(x, kind):
    """(codes as numbers, fp32 scales) of x [..., dh], float64: the definition, one rounding from the exact quotient."""
    amax = np.abs(x).max(-1)
    bad = ~np.isfinite(amax)
    scale = (np.where(bad, 0, amax) / QMAX[kind]).astype(np.float32)
    q = np.where(bad[..., None], 0, x) / np.where(scale == 0, 1, scale).astype(np.float64)[..., None]
    q = np.where((scale == 0)[..., None], 0, q)
    if kind == torch.int8:
        code = np.clip(np.rint(q), -127, 127)
    else:
        mid = (E4M3[1:] + E4M3[:-1]) / 2
        lo, hi = np.searchsorted(mid, np.abs(q), "left"), np.searchsorted(mid, np.abs(q), "right")
        code = E4M3[np.where(lo % 2 == 0, lo, hi)] * np.sign(q)
    return code, np.where(bad, np.float32("nan"), scale)


class Pool:
    """Pools full of values nobody may use (NaN where the type has one), and a page table in random order."""

    def __init__(self, kind, n_seq, tokens, Hkv, dh, page, seed=0, spare=2, n_pages=None):
        self.kind, self.page, self.n_seq = kind, page, n_seq
        per = max(1, -(-tokens // page))
        used = n_seq * per
        n_pages = n_pages or used + spare
        shape = (n_pages, Hkv, page, dh)
        g = torch.Generator().manual_seed(seed)
        if kind == torch.bfloat16:
            mk = lambda: torch.full(shape, float("nan"), dtype=kind, device=DEV)
            self.ks = self.vs = None
        else:
            mk = lambda: torch.full(shape, 0x7f if kind != torch.int8 else -128, dtype=torch.uint8 if kind != torch.int8 else torch.int8, device=DEV).view(kind)
            self.ks, self.vs = (torch.full(shape[:3], float("nan"), device=DEV) for _ in range(2))
        self.k, self.v = mk(), mk()
        self.table = (n_pages - 1 - torch.randperm(used + min(spare, n_pages - used), generator=g)[:used]).to(torch.int32).reshape(n_seq, per)
        self.dev_table = self.table.to(DEV)
        self.raw()

    def raw(self):
        self.cache = SL.PagedKV(self.k, self.v, self.dev_table, self.ks, self.vs)

    def rows(self, pool, b, n):
        """[n][Hkv][dh] (or [n][Hkv] of scales) of sequence b, on the CPU."""
        pages = self.table[b].long()
        x = pool.view(torch.uint8) if pool.element_size() == 1 else pool
        x = torch.stack([x[int(p)] for p in pages]).cpu()
        x = x.view(pool.dtype) if pool.element_size() == 1 else x
        x = x.to(torch.float32) if pool.element_size() < 4 else x
        return x.transpose(1, 2).reshape(-1, *([x.shape[1]] + list(x.shape[3:])))[:n].double().numpy()

    def values(self, which, b, n):
        pool, scale = (self.k, self.ks) if which == "k" else (self.v, self.vs)
        x = self.rows(pool, b, n)
        return x if scale is None else x * self.rows(scale, b, n)[..., None]


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _write(pool, k, v, idx, N, status=None, n=None, k_dev=None):
    SL.surelock_kv_scatter_paged(pool.cache, k, v, _i32(idx), _i32([len(idx) if n is None else n]), N, status)


# ---- refusals, without a GPU ------------------------------------------------------------------------------------------
def _raw_cache(**over):
    d = dict(k=0x1000, v=0x2000, k_scale=0x3000, v_scale=0x4000, page_table=0x5000, n_pages=4, page_size=64, max_pages=2, n_kv_heads=2,
             head_dim=128, dtype=SL.SL_E4M3)
    d.update(over)
    return SL._PagedKV(*[d[n] for n, _ in SL._PagedKV._fields_])


BAD_CACHES = [(dict(k=None), -1), (dict(v=None), -1), (dict(page_table=None), -1), (dict(k_scale=None), -1), (dict(v_scale=None), -1),
              (dict(n_pages=0), -1), (dict(max_pages=0), -1), (dict(n_kv_heads=0), -1), (dict(dtype=SL.SL_FP32), -1), (dict(dtype=9), -1),
              (dict(page_size=8), -5), (dict(page_size=48), -5), (dict(page_size=512), -5), (dict(page_size=0), -5), (dict(head_dim=96), -5),
              (dict(k=0x1008), -5), (dict(v_scale=0x4004), -5), (dict(max_pages=1 << 30), -5)]


@pytest.mark.parametrize("over,rc", BAD_CACHES)
def test_bad_caches_are_refused_on_the_host(over, rc):
    build_mod.build()
    L = SL.lib()
    c = ctypes.byref(_raw_cache(**over))
    assert L.surelock_kv_scatter_paged(c, 0x100, 0x200, 256, 0x300, 0x400, 3, 1, 100, SL.SL_BF16, None, None) == rc
    assert L.surelock_kv_gather_paged(c, 0x300, 0x400, 3, 1, 100, 0x100, 0x200, 256, SL.SL_BF16, None, None) == rc
    assert L.surelock_attention_paged(c, 0x100, 512, 0x200, 0x300, 3, 1, 4, 0x400, 512, 0x500, None, None) == rc


def test_bad_arguments_are_refused_on_the_host():
    build_mod.build()
    L = SL.lib()
    c = ctypes.byref(_raw_cache())
    good = [c, 0x100, 0x200, 256, 0x300, 0x400, 3, 1, 100, SL.SL_BF16, None, None]
    for at, value, rc in [(1, None, -1), (2, None, -1), (4, None, -1), (5, None, -1), (6, -1, -1), (7, 0, -1), (8, 0, -1), (9, SL.SL_INT8, -1),
                          (3, 255, -1), (3, 260, -5), (1, 0x108, -5), (0, None, -1)]:
        bad = list(good)
        bad[at] = value
        assert L.surelock_kv_scatter_paged(*bad) == rc, (at, value)
    good = [c, 0x100, 512, 0x200, 0x300, 3, 1, 4, 0x400, 512, 0x500, None, None]
    for at, value, rc in [(0, None, -1), (1, None, -1), (3, None, -1), (4, None, -1), (8, None, -1), (10, None, -1), (5, -1, -1), (6, 0, -1),
                          (7, 0, -1), (7, 3, -1), (2, 511, -1), (9, 511, -1), (2, 516, -5), (1, 0x108, -5), (10, 0x508, -5), (6, 1025, -5), (5, 0, 0)]:
        bad = list(good)
        bad[at] = value
        assert L.surelock_attention_paged(*bad) == rc, (at, value)
    assert L.surelock_attention_paged_workspace_bytes(96) == 0


def test_binding_refuses_what_it_can_see():
    t = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(SL.SurelockError):                             # not on a CUDA device
        SL.PagedKV(t, t, torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(SL.SurelockError):                             # scales without an 8-bit type
        SL.PagedKV(t, t, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(2, 1, 16), torch.zeros(2, 1, 16))
    with pytest.raises(SL.SurelockError):                             # and an 8-bit type without scales
        SL.PagedKV(t.to(torch.int8), t.to(torch.int8), torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(SL.SurelockError):
        SL.PagedKV(t.double(), t.double(), torch.zeros(1, 2, dtype=torch.int32))


# ---- writing and reading back -----------------------------------------------------------------------------------------
gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh,Hkv,page,dtype", [(128, 2, 64, torch.bfloat16), (64, 5, 16, torch.float32), (64, 1, 256, torch.bfloat16),
                                               (128, 3, 32, torch.float32), (128, 8, 128, torch.bfloat16)])
def test_written_codes_are_exact_and_come_back(kind, dh, Hkv, page, dtype):
    B, N = 2, 150
    g = torch.Generator().manual_seed(dh + page)
    idx = sorted(torch.randperm(B * N, generator=g)[:101].tolist())
    M = len(idx)
    x = [torch.randn(M + 2, Hkv, dh, generator=g) * torch.exp(2 * torch.randn(M + 2, Hkv, 1, generator=g)) for _ in range(2)]
    for t in x:
        t[0, 0] = 0                                                   # all zero
        t[1, 0, :] = 2.0 ** -120                                      # tiny, equal
        t[2, 0] *= 2.0 ** -125                                        # subnormal scales
        t[3, 0] = torch.arange(dh) - dh / 2 + 0.5                     # many values on borders (scale below)
        t[3, 0, 0] = 127.0
        t[4, 0] = (torch.arange(dh) % 17) / 16 - 0.5                  # quotients with few bits
        t[4, 0, 0] = 448.0
        t[5, 0, 3] = float("inf")
        t[6, 0, 5] = float("nan")
        t[7, 0] *= 1e37
        t[8, 0] = -3.0
    dt = [t.to(dtype).to(DEV) for t in x]
    pool = Pool(kind, B, N, Hkv, dh, page)
    before = [pool.k.clone(), pool.v.clone()]
    status = _i32([0])
    SL.surelock_kv_scatter_paged(pool.cache, dt[0], dt[1], _i32(idx + [0, 1]), _i32([M]), N, status)
    assert status.item() == 0
    for b in range(B):
        at = [i for i, f in enumerate(idx) if f // N == b]
        place = [idx[i] % N for i in at]
        for t, p, s in ((dt[0], pool.k, pool.ks), (dt[1], pool.v, pool.vs)):
            want = t[at].cpu().double().numpy()
            got = pool.rows(p, b, N)
            if kind == torch.bfloat16:
                assert np.array_equal(got[place], t[at].cpu().to(torch.bfloat16).double().numpy(), equal_nan=True)
                continue
            code, scale = quantise(want, kind)
            got_scale = pool.rows(s, b, N)
            assert np.array_equal(got_scale[place].astype(np.float32), scale, equal_nan=True)
            assert np.array_equal(got[place], code)
    # what was not named keeps its bytes
    named = {(int(pool.table[f // N, f % N // page]), f % N % page) for f in idx}
    keep = torch.ones(pool.k.shape[0], page, dtype=torch.bool)
    for p, i in named:
        keep[p, i] = False
    for now, was in zip((pool.k, pool.v), before):
        raw = lambda t: (t.view(torch.uint8) if t.element_size() == 1 else t.view(torch.int16)).transpose(1, 2)[keep.to(DEV)]
        assert torch.equal(raw(now), raw(was))
    # and back, in another order, some twice
    order = torch.randperm(M, generator=g)[: M - 5].tolist() + [3, 3, 8]
    for out_t in (torch.bfloat16, torch.float32):
        out = [torch.full((len(order) + 1, Hkv, dh), 7.0, dtype=out_t, device=DEV) for _ in range(2)]
        SL.surelock_kv_gather_paged(pool.cache, _i32([idx[i] for i in order] + [0]), _i32([len(order)]), N, out[0], out[1], status)
        assert status.item() == 0
        for o, which in zip(out, ("k", "v")):
            vals = [pool.values(which, b, N) for b in range(B)]
            want = np.stack([vals[idx[i] // N][idx[i] % N] for i in order])
            want = torch.from_numpy(want).to(torch.float32).to(out_t)  # 11 + 24 bits: one rounding to fp32, one to bf16
            assert torch.equal(o[:-1].cpu().nan_to_num(nan=123.0), want.nan_to_num(nan=123.0))
            assert torch.all(o[-1] == 7.0)


@gpu
@pytest.mark.parametrize("kind", KINDS[1:])
def test_codes_next_to_borders(kind):
    """fp32 values a step or two on both sides of every border between two codes."""
    dh, Q = 128, QMAX[kind]
    amax = np.float32(3.7)
    s = np.float32(amax / Q)
    grid = np.arange(0, 128.0) if kind == torch.int8 else E4M3
    mid = ((grid[1:] + grid[:-1]) / 2 * np.float64(s)).astype(np.float32)
    vals = np.concatenate([mid, np.nextafter(mid, np.float32(9)), np.nextafter(mid, np.float32(0)), np.nextafter(np.nextafter(mid, np.float32(9)), np.float32(9))])
    vals = np.concatenate([vals, -vals])
    rows = -(-len(vals) // (dh - 1))
    x = np.zeros((rows, 1, dh), np.float32)
    x[:, 0, 0] = amax
    x[:, 0, 1:].reshape(-1)[:0] = 0
    flat = np.zeros(rows * (dh - 1), np.float32)
    flat[: len(vals)] = vals
    x[:, 0, 1:] = flat.reshape(rows, dh - 1)
    pool = Pool(kind, 1, rows, 1, dh, 16)
    t = torch.from_numpy(x).to(DEV)
    _write(pool, t, t, list(range(rows)), rows)
    code, scale = quantise(x.astype(np.float64), kind)
    assert np.array_equal(pool.rows(pool.ks, 0, rows).astype(np.float32), scale)
    assert np.array_equal(pool.rows(pool.k, 0, rows), code)


@gpu
@pytest.mark.parametrize("kind", KINDS[1:])
def test_every_quotient_of_two_bf16_significands(kind):
    """bf16 rows: every significand of the largest magnitude times every significand of an element, 12 binades down."""
    dh = 128
    m = torch.arange(128, 256, dtype=torch.float64)
    rows = []
    for e, top in ((0, m), (120, m[::9]), (-71, m[::9]), (-76, m[::9])):      # the last two on both sides of 2^-64
        for amax in top:
            x = (m[None] * 2.0 ** -torch.arange(13.0, dtype=torch.float64)[:, None]).reshape(-1)
            x = x[x <= amax]
            x = torch.cat([x, torch.zeros(-len(x) % (dh - 1), dtype=torch.float64)]).reshape(-1, dh - 1)
            x *= 1 - 2 * (torch.arange(dh - 1) % 2)
            rows.append(torch.cat([torch.full((len(x), 1), float(amax), dtype=torch.float64), x], 1) * 2.0 ** e)
    x = torch.cat(rows)[:, None].to(torch.bfloat16)
    n = len(x)
    pool = Pool(kind, 1, n, 1, dh, 256)
    SL.surelock_kv_scatter_paged(pool.cache, x.to(DEV), x.flip(0).to(DEV), torch.arange(n, dtype=torch.int32, device=DEV), _i32([n]), n)
    for t, p, s in ((x, pool.k, pool.ks), (x.flip(0), pool.v, pool.vs)):
        code, scale = quantise(t.double().numpy(), kind)
        assert np.array_equal(pool.rows(s, 0, n).astype(np.float32), scale)
        assert np.array_equal(pool.rows(p, 0, n), code)


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh,Hkv,M,dtype", [(128, 5, 3001, torch.bfloat16), (64, 7, 4201, torch.float32), (128, 33, 701, torch.float32)])
def test_many_rows_of_odd_heads(kind, dh, Hkv, M, dtype):
    """More (row, head) pairs than the SMs hold at once, heads that do not divide evenly, a count below the capacity."""
    n = M - 1
    g = torch.Generator().manual_seed(M)
    k, v = (torch.randn(M, Hkv, dh, generator=g).to(dtype) for _ in range(2))
    idx = torch.randperm(M + 40, generator=g)[:M].to(torch.int32)
    pool = Pool(kind, 1, M + 40, Hkv, dh, 64)
    SL.surelock_kv_scatter_paged(pool.cache, k.to(DEV), v.to(DEV), idx.to(DEV), _i32([n]), M + 40)
    out = [torch.full((M, Hkv, dh), 7.0, device=DEV) for _ in range(2)]
    SL.surelock_kv_gather_paged(pool.cache, idx.to(DEV), _i32([n]), M + 40, out[0], out[1])
    at = idx[:n].long().numpy()
    for t, which, p, s, o in ((k, "k", pool.k, pool.ks, out[0]), (v, "v", pool.v, pool.vs, out[1])):
        got = pool.rows(p, 0, M + 40)
        if kind == torch.bfloat16:
            assert np.array_equal(got[at], t[:n].to(torch.bfloat16).double().numpy())
        else:
            code, scale = quantise(t[:n].double().numpy(), kind)
            assert np.array_equal(got[at], code)
            assert np.array_equal(pool.rows(s, 0, M + 40)[at].astype(np.float32), scale)
        want = torch.from_numpy(pool.values(which, 0, M + 40)[at]).float()
        assert torch.equal(o[:n].cpu(), want) and torch.all(o[n:] == 7.0)
        untouched = np.setdiff1d(np.arange(M + 40), at)
        if kind != torch.int8:
            assert np.all(np.isnan(got[untouched]))
        else:
            assert np.all(got[untouched] == -128)


@gpu
def test_rows_of_a_wider_buffer_and_small_counts():
    """k and v as parts of packed [q | k | v] rows; no row, one row, fewer rows than the capacity."""
    Hkv, dh, M = 4, 64, 9
    qkv = torch.randn(M, 3, Hkv, dh, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    k, v = qkv[:, 1], qkv[:, 2]
    for n in (0, 1, M):
        pool = Pool(torch.int8, 1, 40, Hkv, dh, 16, seed=n)
        before = pool.k.clone()
        idx = [39, 0, 17, 16, 15, 5, 20, 31, 32]
        SL.surelock_kv_scatter_paged(pool.cache, k, v, _i32(idx), _i32([n]), 40)
        if n == 0:
            assert torch.equal(pool.k, before)
            continue
        code, _ = quantise(k[:n].cpu().double().numpy(), torch.int8)
        assert np.array_equal(pool.rows(pool.k, 0, 40)[idx[:n]], code)
        wide = torch.zeros(M, 3, Hkv, dh, device=DEV)
        SL.surelock_kv_gather_paged(pool.cache, _i32(idx), _i32([n]), 40, wide[:, 0], wide[:, 2])
        assert np.array_equal(wide[:n, 0].cpu().double().numpy(), pool.values("k", 0, 40)[idx[:n]].astype(np.float32))
        assert np.array_equal(wide[:n, 2].cpu().double().numpy(), pool.values("v", 0, 40)[idx[:n]].astype(np.float32))
        assert wide[:, 1].abs().max() == 0 and (n == M or wide[n:].abs().max() == 0)


@gpu
def test_bad_positions_and_pages_are_skipped():
    Hkv, dh, N = 2, 64, 48
    pool = Pool(torch.float8_e4m3fn, 2, N, Hkv, dh, 16)
    pool.table[1, 1] = pool.k.shape[0]                                # a page behind the pool
    pool.table[0, 2] = -1
    pool.dev_table.copy_(pool.table)
    x = torch.randn(5, Hkv, dh, generator=torch.Generator().manual_seed(1)).to(DEV)
    before = [pool.k.view(torch.uint8).clone(), pool.v.view(torch.uint8).clone(), pool.ks.clone(), pool.vs.clone()]
    bad = [N + 16, 32, -1, 2 * N, 5 * N]                              # bad pages (2), and no such position (3)
    status = _i32([0])
    _write(pool, x, x, bad, N, status)
    assert status.item() == 4
    for now, was in zip((pool.k.view(torch.uint8), pool.v.view(torch.uint8), pool.ks, pool.vs), before):
        assert torch.equal(now.nan_to_num(), was.nan_to_num())
    status.zero_()
    out = [torch.ones(6, Hkv, dh, device=DEV) for _ in range(2)]
    _write(pool, x[:1], x[:1], [7], N, status)
    assert status.item() == 0
    SL.surelock_kv_gather_paged(pool.cache, _i32(bad + [7]), _i32([6]), N, out[0], out[1], status)
    assert status.item() == 4
    assert out[0][:5].abs().max() == 0 and out[1][:5].abs().max() == 0 and out[0][5].abs().max() > 0
    # positions behind the tables' pages (N larger than they cover)
    status.zero_()
    SL.surelock_kv_gather_paged(pool.cache, _i32([60]), _i32([1]), 1000, out[0][:1], out[1][:1], status)
    assert status.item() == 4


# ---- attention --------------------------------------------------------------------------------------------------------
def _fill(pool, lens, Hkv, dh, seed=0, k_std=1.0, scale_spread=0.0):
    """Random values at every token of every sequence, written by plain indexing."""
    g = torch.Generator().manual_seed(seed)
    for b, n in enumerate(lens):
        for name in ("k", "v"):
            p, sc = (pool.k, pool.ks) if name == "k" else (pool.v, pool.vs)
            x = torch.randn(max(n, 1), Hkv, dh, generator=g) * (k_std if name == "k" else 1.0)
            i = torch.arange(n)
            page, place = pool.table[b, i // pool.page].long().to(DEV), (i % pool.page).to(DEV)
            if sc is None:
                p[page, :, place] = x[:n].to(torch.bfloat16).to(DEV)
                continue
            s = (x.abs().amax(2) / QMAX[pool.kind])
            c = x / s[..., None]
            c = c.round().to(torch.int8) if pool.kind == torch.int8 else c.to(torch.float8_e4m3fn)
            s = s * torch.exp(scale_spread * torch.randn(s.shape, generator=g)) if name == "v" else s
            p.view(torch.uint8)[page, :, place] = c[:n].view(torch.uint8).to(DEV)
            sc[page, :, place] = s[:n].to(DEV)


def _want(pool, q, offs, lens, G):
    """(o, tolerance besides that of rounding o) in float64."""
    dh = q.shape[2]
    o = np.zeros(q.shape)
    A = np.zeros(q.shape)
    c = 2.0 ** -8 if pool.ks is None else 2.0 ** -11
    for b, n in enumerate(lens):
        if n == 0 or offs[b] == offs[b + 1]:
            continue
        k, v = pool.values("k", b, n), pool.values("v", b, n)
        for h in range(q.shape[1]):
            s = q[offs[b]:offs[b + 1], h] @ k[:, h // G].T / np.sqrt(dh)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o[offs[b]:offs[b + 1], h] = p @ v[:, h // G]
            A[offs[b]:offs[b + 1], h] = (c + 2.0 ** -12) * (p @ np.abs(v[:, h // G]))
            if pool.ks is not None:
                W = (p * pool.rows(pool.vs, b, n)[:, h // G]).max(1, keepdims=True)
                A[offs[b]:offs[b + 1], h] += n * QMAX[pool.kind] * 2.0 ** -33 * W
    return o, A


def _attend(pool, q, offs, lens, status=None, ws=None, o=None):
    o = torch.full_like(q, 7.0) if o is None else o
    ws = torch.full((SL.surelock_attention_paged_workspace_bytes(q.shape[2]),), 255, dtype=torch.uint8, device=DEV) if ws is None else ws
    SL.surelock_attention_paged(pool.cache, q, _i32(offs), _i32(lens), o, ws, status)
    return o


def _near(got, o, A, kind):
    tol = 2.0 ** -8 * np.abs(o) + A + 1e-30
    d = np.abs(got.cpu().double().numpy() - o)
    worst = float((d / tol).max()) if d.size else 0.0
    assert np.all(np.isfinite(d)) and worst <= 1.0, worst


ATT = [
    # lens, rows, Hkv, G, page
    ([1], [1], 1, 1, 16),
    ([63], [1], 2, 1, 64),
    ([64, 65, 1, 0, 129], [1, 1, 1, 1, 1], 2, 4, 16),
    ([500], [23], 4, 1, 64),
    ([17, 300, 0, 128], [3, 0, 2, 5], 1, 7, 32),
    ([1000, 3], [1, 70], 2, 2, 128),
    ([4099], [1], 1, 8, 256),
    ([200, 77, 513], [40, 17, 33], 3, 1, 16),
    ([2500], [130], 1, 1, 64),
]


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("lens,rows,Hkv,G,page", ATT)
def test_attention_paged(kind, dh, lens, rows, Hkv, G, page):
    pool = Pool(kind, len(lens), max(lens), Hkv, dh, page, seed=sum(lens))
    _fill(pool, lens, Hkv, dh, seed=len(lens))
    for b, n in enumerate(lens):                                      # entries behind the last token are not read
        pool.dev_table[b, -(-n // page):] = -5
    offs = [0] + np.cumsum(rows).tolist()
    q = (torch.randn(offs[-1] + 2, Hkv * G, dh, generator=torch.Generator().manual_seed(7)) * 2).to(torch.bfloat16).to(DEV)
    status = _i32([0])
    got = _attend(pool, q, offs, lens, status)
    assert status.item() == 0
    o, A = _want(pool, q.cpu().double().numpy(), offs, lens, G)
    _near(got[: offs[-1]], o[: offs[-1]], A[: offs[-1]], kind)
    assert torch.all(got[offs[-1]:] == 7.0)                           # rows behind the last sequence keep their bytes
    for b, n in enumerate(lens):
        if n == 0:
            assert torch.all(got[offs[b]:offs[b + 1]] == 0)
    assert torch.equal(got, _attend(pool, q, offs, lens))             # the same bits again


@gpu
@pytest.mark.parametrize("kind", KINDS)
def test_attention_paged_growing_scores_and_spread_scales(kind):
    """Maxima that grow along the keys (O is rescaled), value scales over ten orders of magnitude, large scores."""
    lens, Hkv, dh, G = [700, 300], 2, 128, 2
    pool = Pool(kind, 2, 700, Hkv, dh, 32)
    _fill(pool, lens, Hkv, dh, seed=5, k_std=4.0, scale_spread=6.0)
    if pool.ks is not None:
        i = torch.arange(700)
        page, place = pool.table[0, i // 32].long().to(DEV), (i % 32).to(DEV)
        pool.ks[page, :, place] *= torch.linspace(0.01, 3.0, 700, device=DEV)[:, None]
        pool.vs[page[100], :, place[100]] = 0.0                       # a token whose values are all zero
        pool.vs[page[300], :, place[300]] = 1e-38
    offs = [0, 5, 6]
    q = (torch.randn(6, Hkv * G, dh, generator=torch.Generator().manual_seed(8)) * 4).to(torch.bfloat16)
    q[0] = 0
    q[1] *= 1e-20
    q = q.to(DEV)
    got = _attend(pool, q, offs, lens)
    o, A = _want(pool, q.cpu().double().numpy(), offs, lens, G)
    _near(got, o, A, kind)


@gpu
def test_attention_paged_strides_streams_and_graphs():
    kind, Hkv, dh, G = torch.float8_e4m3fn, 2, 128, 2
    lens, rows = [333, 90, 640], [2, 1, 9]
    pool = Pool(kind, 3, 640, Hkv, dh, 64)
    _fill(pool, lens, Hkv, dh)
    offs = [0, 2, 3, 12]
    wide = torch.randn(12, 2, Hkv * G, dh, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).to(DEV)
    q = wide[:, 0]
    plain = _attend(pool, q.contiguous(), offs, lens)
    out = torch.full((12, 3, Hkv * G, dh), 7.0, dtype=torch.bfloat16, device=DEV)
    _attend(pool, q, offs, lens, o=out[:, 1])
    assert torch.equal(out[:, 1], plain) and torch.all(out[:, 0] == 7.0) and torch.all(out[:, 2] == 7.0)
    # two calls at once on two streams, each with its own workspace
    d_offs, d_lens = _i32(offs), _i32(lens)
    mk_ws = lambda: torch.empty(SL.surelock_attention_paged_workspace_bytes(dh), dtype=torch.uint8, device=DEV)
    streams, outs, spaces = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(plain) for _ in range(2)], [mk_ws(), mk_ws()]
    qc = q.contiguous()
    torch.cuda.synchronize()
    for _ in range(20):
        for s, o, w in zip(streams, outs, spaces):
            with torch.cuda.stream(s):
                SL.surelock_attention_paged(pool.cache, qc, d_offs, d_lens, o, w)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], plain) and torch.equal(outs[1], plain)
    # captured once, replayed with other lengths and other values in the same buffers
    g, o = torch.cuda.CUDAGraph(), torch.zeros_like(plain)
    with torch.cuda.graph(g):
        SL.surelock_attention_paged(pool.cache, qc, d_offs, d_lens, o, spaces[0])
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, plain)
    d_lens.copy_(_i32([1, 64, 500]))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, _attend(pool, qc, offs, [1, 64, 500]))


@gpu
def test_attention_paged_bad_tables_lengths_and_offsets():
    kind, Hkv, dh, page = torch.int8, 1, 64, 16
    pool = Pool(kind, 2, 64, Hkv, dh, page)
    _fill(pool, [64, 64], Hkv, dh)
    q = torch.randn(4, 2, dh, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    status = _i32([0])
    # a bad page reads as zeros: the same as a page whose scales are zero
    pool.dev_table[1, 2] = 1 << 30
    got = _attend(pool, q, [0, 1, 4], [64, 50], status)
    assert status.item() == 4
    pool.dev_table.copy_(pool.table)
    p = int(pool.table[1, 2])
    keep = pool.ks[p].clone(), pool.vs[p].clone()
    pool.ks[p], pool.vs[p] = 0, 0
    status.zero_()
    assert torch.equal(got, _attend(pool, q, [0, 1, 4], [64, 50], status)) and status.item() == 0
    pool.ks[p], pool.vs[p] = keep
    # lengths out of range are clamped
    full = _attend(pool, q, [0, 1, 4], [64, 0])
    got = _attend(pool, q, [0, 1, 4], [65, -3], status)
    assert status.item() == 4 and torch.equal(got, full) and torch.all(got[1:] == 0)
    # row offsets beyond the rows
    status.zero_()
    got = _attend(pool, q, [0, 1, 9], [64, 64], status)
    assert status.item() == 4 and torch.equal(got, _attend(pool, q, [0, 1, 4], [64, 64]))
    status.zero_()
    got = _attend(pool, q, [0, 4, 1], [64, 64], status)               # a sequence with less than no rows has none
    assert status.item() == 4 and torch.equal(got, _attend(pool, q, [0, 4, 4], [64, 64]))


@gpu
def test_attention_paged_many_sequences():
    B, Hkv, dh = 1024, 1, 64
    lens = [(37 * b) % 90 for b in range(B)]
    pool = Pool(torch.float8_e4m3fn, B, 90, Hkv, dh, 16)
    _fill(pool, [max(lens)] * 4, Hkv, dh)                             # values for the first sequences; all share their pages
    pool.table[4:] = pool.table[torch.arange(4, B) % 4]
    pool.dev_table.copy_(pool.table)
    offs = list(range(B + 1))
    q = torch.randn(B, 2, dh, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(DEV)
    got = _attend(pool, q, offs, lens)
    o, A = _want(pool, q.cpu().double().numpy(), offs, lens, 2)
    _near(got, o, A, pool.kind)


@gpu
def test_offsets_beyond_32_bits():
    """A pool of more than 2^31 codes: pages at its end are written, read back and attended to."""
    Hkv, dh, page = 8, 128, 256
    n_pages = (1 << 31) // (Hkv * dh * page) + 9
    pool = Pool(torch.int8, 1, 400, Hkv, dh, page, spare=1, n_pages=n_pages)
    assert int(pool.table.min()) >= n_pages - 3
    x = [torch.randn(400, Hkv, dh, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16).to(DEV) for i in range(2)]
    idx = list(range(400))
    _write(pool, x[0], x[1], idx, 400)
    code, _ = quantise(x[0].cpu().double().numpy(), torch.int8)
    assert np.array_equal(pool.rows(pool.k, 0, 400), code)
    out = [torch.zeros(400, Hkv, dh, device=DEV) for _ in range(2)]
    SL.surelock_kv_gather_paged(pool.cache, _i32(idx), _i32([400]), 400, out[0], out[1])
    assert np.array_equal(out[1].cpu().double().numpy(), pool.values("v", 0, 400).astype(np.float32))
    q = torch.randn(2, Hkv, dh, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).to(DEV)
    got = _attend(pool, q, [0, 2], [400])
    o, A = _want(pool, q.cpu().double().numpy(), [0, 2], [400], 1)
    _near(got, o, A, pool.kind)


@gpu
def test_refusals_with_tensors(monkeypatch):
    Hkv, dh, N = 2, 64, 48
    pool = Pool(torch.int8, 1, N, Hkv, dh, 16)
    k, v = (torch.randn(3, Hkv, dh, device=DEV) for _ in range(2))
    idx, n = _i32([0, 1, 2]), _i32([3])
    q = torch.randn(3, 4, dh, device=DEV).to(torch.bfloat16)
    offs, lens, ws = _i32([0, 3]), _i32([3]), torch.empty(SL.surelock_attention_paged_workspace_bytes(dh), dtype=torch.uint8, device=DEV)
    write = lambda *a: SL.surelock_kv_scatter_paged(pool.cache, *a)
    read = lambda *a: SL.surelock_kv_gather_paged(pool.cache, *a)
    attend = lambda *a: SL.surelock_attention_paged(pool.cache, *a)
    write(k[:0], v[:0], idx, n, N)                                    # no rows: nothing to do
    read(idx, n, N, k[:0], v[:0])
    attend(q[:0], offs, lens, q[:0], ws)
    good = [(write, (k, v, idx, n, N)), (read, (idx, n, N, k, v)), (attend, (q, offs, lens, q.clone(), ws))]
    for f, a in good:
        f(*a)
        for i, t in enumerate(a):
            if isinstance(t, torch.Tensor):                           # one on the CPU, or of another type
                for bad in (t.cpu(), t.long()) if t.dtype == torch.int32 else (t.cpu(),):
                    with pytest.raises(SL.SurelockError):
                        f(*a[:i], bad, *a[i + 1:])
    for f, a in [(write, (k[:, :1], v[:, :1], idx, n, N)), (write, (k, v[:2], idx, n, N)), (write, (k, v, idx[:2], n, N)), (write, (k, v, idx, n, 0)),
                 (read, (idx, n, N, k.half(), v.half())), (read, (idx, n, N, k[:1].expand(3, Hkv, dh), v[:1].expand(3, Hkv, dh))),
                 (attend, (q[:, :3], offs, lens, q[:, :3], ws)), (attend, (q, offs, lens, q, ws[:100])), (attend, (q, offs, _i32([1, 1]), q, ws)),
                 (attend, (q.float(), offs, lens, q.float(), ws))]:
        with pytest.raises(SL.SurelockError):
            f(*a)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)       # as if another device were the current one
    for f, a in good:
        with pytest.raises(SL.SurelockError):
            f(*a)


@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,dh", [([1, 3], 128), ([8, 2], 64), ([12, 9], 128), ([21, 1], 64)])
def test_attention_paged_nan_stays_where_it_is(kind, rows, dh):
    """A NaN in a query spoils that (row, head); one in a token spoils its key head's rows of that sequence; infinities in q too."""
    lens, Hkv, G = [300, 130], 2, 2
    pool = Pool(kind, 2, 300, Hkv, dh, 32)
    _fill(pool, lens, Hkv, dh, seed=3)
    offs = [0] + np.cumsum(rows).tolist()
    q = torch.randn(offs[-1], Hkv * G, dh, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16)
    o, A = _want(pool, q.double().numpy(), offs, lens, G)

    def check(got, spoilt):
        assert torch.all(torch.isnan(got[spoilt])), "spoilt rows are NaN"
        keep = ~spoilt.numpy()
        _near(got.cpu()[~spoilt], o[keep], A[keep], kind)

    for value in (float("nan"), float("inf")):
        bad = q.clone()
        bad[0, 1, 7] = value
        spoilt = torch.zeros(offs[-1], Hkv * G, dtype=torch.bool)
        spoilt[0, 1] = True
        check(_attend(pool, bad.to(DEV), offs, lens).cpu(), spoilt)
    page, place = int(pool.table[0, 200 // 32]), 200 % 32
    spoilt = torch.zeros(offs[-1], Hkv * G, dtype=torch.bool)
    spoilt[:offs[1], G:] = True                                       # sequence 0, key head 1
    for t in ((pool.k, pool.v) if pool.ks is None else (pool.ks, pool.vs)):
        was = t[page, 1, place].clone()
        t[page, 1, place] = float("nan")
        check(_attend(pool, q.to(DEV), offs, lens).cpu(), spoilt)
        t[page, 1, place] = was


# ---- rows whose scores are all minus infinity -------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("lens,rows,Hkv,G,tokens", [
    ([1, 2, 0], [1, 2, 1], 2, 2, 64),                                 # tiles of 8 rows, whole items
    ([300, 0, 64], [1, 2, 1], 2, 2, 300),                             # cut into a few pieces
    ([2500, 1], [1, 1], 1, 4, 2500),                                  # and into many
    ([1, 2, 0], [9, 13, 5], 2, 1, 64),                                # tiles of 16
    ([300, 0, 2000], [9, 13, 5], 1, 1, 2000),
    ([1, 0], [20, 21], 8, 1, 2048),                                   # tiles of 32
    ([600, 2], [20, 21], 8, 1, 2048),
])
def test_scores_of_minus_infinity_give_nan_and_no_key_gives_zeros(kind, lens, rows, Hkv, G, tokens):
    """softmax over scores that are all -inf is 0 / 0; only a sequence without keys has rows of zeros."""
    dh = 128
    pool = Pool(kind, len(lens), tokens, Hkv, dh, 32)
    _fill(pool, lens, Hkv, dh, seed=sum(lens))
    if kind == torch.bfloat16:
        pool.k[..., 7] = -1.0
    else:
        pool.k.view(torch.uint8)[..., 7] = 0xb8 if kind != torch.int8 else 251      # -1, -5
    offs = [0] + np.cumsum(rows).tolist()
    q = torch.randn(offs[-1], Hkv * G, dh, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16)
    o, A = _want(pool, q.double().numpy(), offs, lens, G)
    spoilt = torch.zeros(offs[-1], Hkv * G, dtype=torch.bool)
    for b in range(len(lens)):
        spoilt[offs[b], 0] = spoilt[offs[b + 1] - 1, -1] = True
    bad = q.clone()
    bad[..., 7] = torch.where(spoilt, float("inf"), bad[..., 7])
    status = _i32([0])
    got = _attend(pool, bad.to(DEV), offs, lens, status).cpu()
    assert status.item() == 0
    for b, n in enumerate(lens):
        at = slice(offs[b], offs[b + 1])
        if n == 0:
            assert torch.all(got[at] == 0)
            continue
        assert torch.all(torch.isnan(got[at][spoilt[at]]))
        keep = ~spoilt[at]
        _near(got[at][keep], o[at][keep.numpy()], A[at][keep.numpy()], kind)


@gpu
@pytest.mark.parametrize("offs,same", [([0, 2, -2 ** 31], [0, 2, 2]), ([0, 2, 2 ** 31 - 1], [0, 2, 4]), ([-2 ** 31, 2, 4], [0, 2, 4]),
                                       ([2 ** 31 - 1, -2 ** 31, 3], [0, 0, 3]), ([0, 0, -1], [0, 0, 0]), ([2 ** 31 - 1, 2 ** 31 - 1, -2 ** 31], [4, 4, 4])])
def test_row_offsets_of_any_value_are_clamped(offs, same):
    """A difference of two offsets may pass 32 bits; rows that no sequence has left keep their bytes."""
    pool = Pool(torch.int8, 2, 64, 1, 64, 16)
    _fill(pool, [64, 50], 1, 64)
    q = torch.randn(4, 2, 64, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    status = _i32([0])
    got = _attend(pool, q, offs, [64, 50], status)
    assert status.item() == 4 and torch.equal(got, _attend(pool, q, same, [64, 50]))


@gpu
@pytest.mark.parametrize("kind", KINDS[1:])
def test_fp32_codes_next_to_borders_at_every_size(kind):
    """Values up to two steps on both sides of every border between two codes, for largest magnitudes whose quotient by the
    largest code is exact, rounded up and rounded down, on both sides of 2^-64, next to the largest fp32 number, and with subnormal scales."""
    dh, Q = 128, QMAX[kind]
    up, down = lambda x: np.nextafter(x, np.float32(np.inf)), lambda x: np.nextafter(x, np.float32(0))
    f = np.float32
    tops = [f(Q), f(Q * 1.5), f(Q * 2.0 ** -40), f(3.7), f(1.0), f(0.3), f(7.1), f(1e-5), f(12345.678), f(2.0 ** -64), up(f(2.0 ** -64)), down(f(2.0 ** -64)),
            f(3e-20), f(6e-20), f(1e-30), f(1e-36), f(1e-37), f(3e-38), f(2.0 ** -130), f(1e38), down(f(np.inf)), f(2.0 ** 127)]
    exact = [float(t) - Q * float(f(float(t) / Q)) for t in tops]
    assert any(r == 0 for r in exact) and any(r > 0 for r in exact) and any(r < 0 for r in exact)
    grid = np.arange(0, 128.0) if kind == torch.int8 else E4M3
    rows = []
    for amax in tops:
        s = f(float(amax) / Q)
        mid = ((grid[1:] + grid[:-1]) / 2 * np.float64(s)).astype(f)
        vals = np.concatenate([mid, up(mid), down(mid), up(up(mid)), down(down(mid))])
        vals = np.minimum(np.concatenate([vals, -vals]), amax)
        x = np.zeros((-(-len(vals) // (dh - 1)), dh), f)
        flat = np.zeros(len(x) * (dh - 1), f)
        flat[: len(vals)] = vals
        x[:, 0], x[:, 1:] = amax, flat.reshape(len(x), dh - 1)
        rows.append(np.maximum(x, -amax))
    x = np.concatenate(rows)[:, None]
    n = len(x)
    pool = Pool(kind, 1, n, 1, dh, 16)
    k, v = torch.from_numpy(x).to(DEV), torch.from_numpy(x[::-1].copy()).to(DEV)
    _write(pool, k, v, list(range(n)), n)
    for t, p, sc in ((x, pool.k, pool.ks), (x[::-1], pool.v, pool.vs)):
        code, scale = quantise(t.astype(np.float64), kind)
        assert np.array_equal(pool.rows(sc, 0, n).astype(np.float32), scale)
        assert np.array_equal(pool.rows(p, 0, n), code)


# ---- weights of the last product ----------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("lens,rows,Hkv,G,tokens", [
    ([2, 3, 4, 5, 6, 7, 8, 70], [2] * 8, 4, 4, 70),                   # tiles of 8 rows
    ([2, 3, 5, 40], [16] * 4, 2, 1, 40),                              # of 16
    ([2, 3, 5, 7, 300], [32] * 5, 8, 1, 2048),                        # of 32
])
def test_attention_over_bf16_pages_keeps_sixteen_bits_of_a_weight(dh, lens, rows, Hkv, G, tokens):
    """Few keys of either sign, so that results are small beside sum p |v|: the weights enter the product as two bf16 terms, the
    second off by half a step (2^-8) of a residual of at most half a step (2^-8) of the weight."""
    pool = Pool(torch.bfloat16, len(lens), tokens, Hkv, dh, 64)
    _fill(pool, lens, Hkv, dh, seed=dh)
    offs = [0] + np.cumsum(rows).tolist()
    q = torch.randn(offs[-1], Hkv * G, dh, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    got = _attend(pool, q, offs, lens)
    o, A = _want(pool, q.cpu().double().numpy(), offs, lens, G)
    _near(got, o, A * (2.0 ** -16 + 2.0 ** -12) / (2.0 ** -8 + 2.0 ** -12), pool.kind)
