"""The quantised operators together, as one attention block of a served model uses them: 4-bit products for q, k and v, the new
rows written into a paged 8-bit cache, attention over it, and the 4-bit output product added to the residual stream; first a
prompt, then single tokens, eagerly and as a replayed graph.  Every operator is checked in its own file; here each stage is
held against a plain statement in 64 bits of what the stage before it left in memory, with the same bounds, so that a wrong
hand-over (order, layout, count, stream) shows as more than a rounding."""
import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL

from .test_gemm_quantized import _tol, _weights
from .test_paged_kv import DEV, Pool, _attend, _fill, _i32, _near, _want, quantise

pytestmark = pytest.mark.gpu


class Block:
    """d_model 512, 4 query heads on 2 key heads of 128, three sequences on pages of 16."""
    d, H, Hkv, dh, B, N, group = 512, 4, 2, 128, 3, 90, 64

    def __init__(self, kind):
        self.kind = kind
        qkv = (self.H + 2 * self.Hkv) * self.dh
        self.Wqkv, self.wqkv = _weights(qkv, self.d, self.group, True, torch.bfloat16, seed=1)
        self.Wo, self.wo = _weights(self.d, self.H * self.dh, self.group, False, torch.float32, seed=2)
        self.pool = Pool(kind, self.B, self.N, self.Hkv, self.dh, 16)
        self.lens = [0] * self.B
        self.status = _i32([0])

    def buffers(self, M):
        """Device buffers of a step with at most M rows."""
        z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device=DEV)
        return dict(x=z(M, self.d), qkv=z(M, self.wqkv.shape[0]), o=z(M, self.H * self.dh), res=z(M, self.d, t=torch.float32),
                    idx=_i32([0] * M), n=_i32([M]), offs=_i32([0] * (self.B + 1)), lens=_i32([0] * self.B),
                    ws=z(SL.surelock_attention_paged_workspace_bytes(self.dh), t=torch.uint8))

    def launch(self, t):
        """The step's six calls on the current stream."""
        SL.surelock_gemm_quantized(t["x"], self.Wqkv, t["qkv"], t["n"], dev_status=self.status)
        heads = t["qkv"].view(-1, self.H + 2 * self.Hkv, self.dh)
        k, v = heads[:, self.H:self.H + self.Hkv], heads[:, self.H + self.Hkv:]
        SL.surelock_kv_scatter_paged(self.pool.cache, k, v, t["idx"], t["n"], self.N, self.status)
        SL.surelock_attention_paged(self.pool.cache, heads[:, :self.H], t["offs"], t["lens"], t["o"].view(-1, self.H, self.dh), t["ws"], self.status)
        SL.surelock_gemm_quantized(t["o"], self.Wo, t["res"], t["n"], epilogue=1, dev_status=self.status)

    def fill(self, t, new, seed):
        """`new` tokens more for every sequence: inputs and the step's indices; returns the row offsets."""
        g = torch.Generator().manual_seed(seed)
        M = sum(new)
        t["x"][:M] = torch.randn(M, self.d, generator=g).to(torch.bfloat16).to(DEV)
        t["res"].copy_(torch.randn(t["res"].shape, generator=g))
        idx = [b * self.N + self.lens[b] + i for b in range(self.B) for i in range(new[b])]
        self.lens = [have + m for have, m in zip(self.lens, new)]
        offs = [0] + np.cumsum(new).tolist()
        t["idx"][:M] = _i32(idx)
        t["n"].fill_(M)
        t["offs"].copy_(_i32(offs))
        t["lens"].copy_(_i32(self.lens))
        return idx, offs

    def check(self, t, before, idx, offs):
        """Every stage against what the one before it left."""
        M = offs[-1]
        np64 = lambda x: x.cpu().double().numpy()
        x, qkv, o = np64(t["x"][:M]), np64(t["qkv"][:M]), np64(t["o"][:M])
        tol = _tol(x, self.wqkv, self.d, self.group) + 2.0 ** -8 * np.abs(x @ self.wqkv.T)
        assert np.all(np.abs(qkv - x @ self.wqkv.T) <= tol)
        heads = qkv.reshape(M, self.H + 2 * self.Hkv, self.dh)
        for part, p, s in ((heads[:, self.H:self.H + self.Hkv], self.pool.k, self.pool.ks), (heads[:, self.H + self.Hkv:], self.pool.v, self.pool.vs)):
            for b in range(self.B):
                rows = range(offs[b], offs[b + 1])
                place = [idx[r] % self.N for r in rows]
                got = self.pool.rows(p, b, self.N)[place]
                if s is None:
                    assert np.array_equal(got, part[rows])
                else:
                    code, scale = quantise(part[rows], self.kind)
                    assert np.array_equal(got, code) and np.array_equal(self.pool.rows(s, b, self.N)[place].astype(np.float32), scale)
        want, A = _want(self.pool, heads[:, :self.H], offs, self.lens, self.H // self.Hkv)
        _near(t["o"][:M].view(M, self.H, self.dh), want, A, self.kind)
        res = np64(before[:M]) + o @ self.wo.T
        d = np.abs(np64(t["res"][:M]) - res)
        assert np.all(d <= _tol(o, self.wo, self.H * self.dh, self.group) + 2.0 ** -24 * np.abs(res))
        assert torch.equal(t["res"][M:], before[M:]) and self.status.item() == 0


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float8_e4m3fn, torch.int8])
def test_prompt_and_single_tokens(kind):
    block = Block(kind)
    t = block.buffers(80)
    for seed, new in enumerate([(41, 17, 5), (0, 20, 33)]):           # 63 rows, then a longer prompt for two of them
        idx, offs = block.fill(t, new, seed)
        before = t["res"].clone()
        block.launch(t)
        block.check(t, before, idx, offs)
    # single tokens, captured once; a sequence that has ended contributes no row
    t = block.buffers(block.B)
    torch.cuda.synchronize()
    keep = [block.pool.k.clone(), block.pool.v.clone()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.launch(t)
    raw = lambda x: x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16)
    assert all(torch.equal(raw(a), raw(b)) for a, b in zip(keep, (block.pool.k, block.pool.v)))
    for seed, new in enumerate([(1, 1, 1), (1, 0, 1), (1, 1, 1), (0, 0, 0), (0, 1, 1)]):
        idx, offs = block.fill(t, new, 10 + seed)
        before = t["res"].clone()
        graph.replay()
        torch.cuda.synchronize()
        block.check(t, before, idx, offs)


@pytest.mark.parametrize("kind", [torch.float8_e4m3fn, torch.int8])
def test_read_back_into_a_contiguous_cache(kind):
    """Pages read back into [B][N] rows serve the framework's own attention: the same answer from both, within the roundings of
    K and V to bf16 (2^-8 of a score's sum |q||k| / sqrt(d), 2^-8 of the values) and of either result."""
    B, N, H, dh, M = 2, 64, 2, 128, 6
    pool = Pool(kind, B, N, H, dh, 32)
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(B * N, H, dh, generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    every = torch.arange(B * N, dtype=torch.int32, device=DEV)
    SL.surelock_kv_scatter_paged(pool.cache, k, v, every, _i32([B * N]), N)
    kc, vc = (torch.zeros(B * N, H, dh, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    SL.surelock_kv_gather_paged(pool.cache, every, _i32([B * N]), N, kc, vc)
    offs, idx = [0, 2, M], _i32([3, 9, N, N + 1, N + 20, N + 63])
    q = torch.randn(M, H, dh, generator=g).to(torch.bfloat16).to(DEV)
    contiguous, paged = torch.zeros_like(q), torch.zeros_like(q)
    SL.surelock_attention(q, kc, vc, idx, _i32(offs), _i32([M]), B, N, contiguous)
    ws = torch.empty(SL.surelock_attention_paged_workspace_bytes(dh), dtype=torch.uint8, device=DEV)
    SL.surelock_attention_paged(pool.cache, q, _i32(offs), _i32([N, N]), paged, ws)
    for b in range(B):
        kb, vb = pool.values("k", b, N), pool.values("v", b, N)
        for h in range(H):
            rows = range(offs[b], offs[b + 1])
            qh = q[rows, h].cpu().double().numpy()
            s = qh @ kb[:, h].T / np.sqrt(dh)
            p = np.exp(s - s.max(1, keepdims=True))
            p /= p.sum(1, keepdims=True)
            o, spread = p @ vb[:, h], p @ np.abs(vb[:, h])
            ds = 2.0 ** -8 * (np.abs(qh) @ np.abs(kb[:, h]).T / np.sqrt(dh)).max(1, keepdims=True)
            # a score off by ds moves a weight by a factor exp(2 ds) at most; then the rounding of weights, values and result
            tol = (np.exp(2 * ds) - 1 + 2 * 2.0 ** -8 + 2.0 ** -11) * spread + 2.0 ** -8 * np.abs(o)
            for got in (contiguous, paged):
                assert np.all(np.abs(got[rows, h].cpu().double().numpy() - o) <= tol)


# ---- failure detection: a copy that never arrives --------------------------------------------------------------------
@pytest.mark.parametrize("M,n,K,group", [(5, 600, 1024, 64), (13, 5003, 4096, 128), (70, 200, 1056, 32), (128, 300, 4096, 128)])
def test_a_lost_copy_ends_a_product_with_a_status(M, n, K, group):
    """Calls of both kernels, with stages that all fit the ring and with more: the bounded waits run out, status 2 is stored, and
    the next call on the same workspace is right, bit for bit."""
    W, _ = _weights(n, K, group, True, torch.bfloat16, seed=1)
    A = torch.randn(M, K, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    want, got = (torch.zeros(M, n, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ws = torch.full((SL.surelock_gemm_quantized_workspace_bytes(M, K),), 255, dtype=torch.uint8, device=DEV)
    status, count = _i32([0]), _i32([M])
    call = lambda out: SL.surelock_gemm_quantized(A, W, out, count, workspace=ws, dev_status=status)
    call(want)
    assert status.item() == 0
    SL.surelock_lose_next_copy()
    call(got)
    assert status.item() == 2
    assert torch.equal(got[:, -8:], want[:, -8:])                     # features of another CTA than the first
    status.zero_()
    call(got)
    assert status.item() == 0 and torch.equal(got, want)


@pytest.mark.parametrize("kind,lens,rows", [(torch.int8, [64, 200], [1, 2]), (torch.bfloat16, [5000, 100], [1, 1]), (torch.float8_e4m3fn, [3000, 900], [20, 9])])
def test_a_lost_copy_ends_an_attention_with_a_status(kind, lens, rows):
    Hkv, dh = 2, 128
    pool = Pool(kind, 2, max(lens), Hkv, dh, 64)
    _fill(pool, lens, Hkv, dh)
    offs = [0] + np.cumsum(rows).tolist()
    q = torch.randn(offs[-1], Hkv, dh, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    ws = torch.full((SL.surelock_attention_paged_workspace_bytes(dh),), 255, dtype=torch.uint8, device=DEV)
    status = _i32([0])
    want = _attend(pool, q, offs, lens, status, ws)
    assert status.item() == 0
    SL.surelock_lose_next_copy()
    got = _attend(pool, q, offs, lens, status, ws)
    assert status.item() == 3
    assert torch.equal(got[-1, -1], want[-1, -1])                     # of the last sequence and head, far from the first CTA
    status.zero_()
    got = _attend(pool, q, offs, lens, status, ws)
    assert status.item() == 0 and torch.equal(got, want)


@pytest.mark.parametrize("K", [32 * i for i in (1, 8, 9, 16, 24, 40, 57, 130)])
def test_no_wait_runs_to_its_limit_when_a_kernel_leaves(K):
    """Before a CTA leaves it waits for its copies and matrix instructions, at most 2 s and without a status: a wait for the wrong
    phase would show as time only.  Numbers of stages below, at and above the rings' sizes, both kernels, odd and even steps."""
    lens = [K, 3 * K]
    pool = Pool(torch.int8, 2, 3 * K, 1, 64, 16)
    _fill(pool, lens, 1, 64)
    ws = torch.empty(SL.surelock_attention_paged_workspace_bytes(64), dtype=torch.uint8, device=DEV)
    calls = []
    for M, n in ((3, 70), (20, 4800), (40, 130), (128, 300)):
        for group in (32, 64, 128):
            if K % group:
                continue
            W, _ = _weights(n, K, group, True, torch.bfloat16, seed=1)
            A, out = torch.ones(M, K, dtype=torch.bfloat16, device=DEV), torch.zeros(M, n, dtype=torch.bfloat16, device=DEV)
            calls.append(lambda A=A, W=W, out=out, n=_i32([M]): SL.surelock_gemm_quantized(A, W, out, n))
    for rows in ([1, 1], [9, 8], [40, 2]):
        q, offs = torch.ones(sum(rows), 2, 64, dtype=torch.bfloat16, device=DEV), _i32([0, rows[0], sum(rows)])
        calls.append(lambda q=q, offs=offs, o=torch.zeros_like(q), n=_i32(lens): SL.surelock_attention_paged(pool.cache, q, offs, n, o, ws))
    for call in calls:
        call()                                                        # loads the kernel
        t = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        torch.cuda.synchronize()
        t[0].record()
        call()
        t[1].record()
        torch.cuda.synchronize()
        assert t[0].elapsed_time(t[1]) < 100


@pytest.mark.parametrize("M,n,K,group,epilogue", [(5, 600, 4096, 64, 0), (13, 200, 1024, 32, 1), (29, 5003, 1024, 128, 2), (70, 200, 2048, 32, 1),
                                                  (128, 300, 4096, 128, 0), (128, 300, 4096, 64, 2)])
def test_no_feature_keeps_an_incomplete_sum(M, n, K, group, epilogue):
    """K is split over CTAs whose sums meet: what the one that gave up was to contribute to is NaN, without a status too."""
    W, _ = _weights(n, K, group, True, torch.float32, seed=1)
    W2, _ = _weights(n, K, group, True, torch.float32, seed=2)
    A = torch.randn(M, K, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    out = lambda: torch.ones(M, n, dtype=torch.float32 if epilogue == 1 else torch.bfloat16, device=DEV)
    call = lambda c: SL.surelock_gemm_quantized(A, W, c, _i32([M]), epilogue, W2 if epilogue == 2 else None)
    want, got = out(), out()
    call(want)
    SL.surelock_lose_next_copy()
    call(got)
    rows, first = min(M, 64 if group == 32 else 128), 64 if epilogue == 2 else 128   # of a CTA
    assert torch.all(torch.isnan(got[:rows, :first])) and torch.equal(got[:, first:], want[:, first:]) and torch.equal(got[rows:], want[rows:])


@pytest.mark.parametrize("kind,rows", [(torch.int8, [1]), (torch.bfloat16, [1]), (torch.float8_e4m3fn, [12]), (torch.bfloat16, [13])])
def test_no_row_keeps_an_incomplete_softmax(kind, rows):
    """A long sequence whose pieces are joined: without one piece its rows are NaN, those of the other key head as they were."""
    Hkv, dh, lens = 2, 128, [40000]
    pool = Pool(kind, 1, lens[0], Hkv, dh, 256)
    _fill(pool, lens, Hkv, dh)
    offs = [0, rows[0]]
    q = torch.randn(rows[0], Hkv, dh, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    ws = torch.zeros(SL.surelock_attention_paged_workspace_bytes(dh), dtype=torch.uint8, device=DEV)
    want = _attend(pool, q, offs, lens, ws=ws)
    SL.surelock_lose_next_copy()
    got = _attend(pool, q, offs, lens, ws=ws)                         # the workspace holds the pieces of the call before
    assert torch.all(torch.isnan(got[:, 0])) and torch.equal(got[:, 1], want[:, 1])


@pytest.mark.parametrize("status", [torch.zeros(1, dtype=torch.uint8), torch.zeros(1), torch.zeros(2, dtype=torch.int64), torch.zeros(0, dtype=torch.int32)])
def test_a_status_that_is_not_an_int32_word_is_refused(status):
    status = status.to(DEV)
    pool = Pool(torch.int8, 1, 32, 1, 64, 16)
    k = torch.randn(2, 1, 64, device=DEV)
    q, ws = k.to(torch.bfloat16), torch.empty(SL.surelock_attention_paged_workspace_bytes(64), dtype=torch.uint8, device=DEV)
    W, _ = _weights(40, 128, 64, False, torch.bfloat16, seed=1)
    A, C = torch.zeros(2, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(2, 40, dtype=torch.bfloat16, device=DEV)
    for call in (lambda s: SL.surelock_kv_scatter_paged(pool.cache, k, k, _i32([0, 1]), _i32([2]), 32, s),
                 lambda s: SL.surelock_kv_gather_paged(pool.cache, _i32([0, 1]), _i32([2]), 32, k, k.clone(), s),
                 lambda s: SL.surelock_attention_paged(pool.cache, q, _i32([0, 2]), _i32([2]), q.clone(), ws, s),
                 lambda s: SL.surelock_gemm_quantized(A, W, C, _i32([2]), dev_status=s)):
        call(_i32([0]))
        with pytest.raises(SL.SurelockError):
            call(status)
