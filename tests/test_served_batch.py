"""The operators of a served batch together, as a program that serves many requests runs them: pages and positions from the requests'
lengths, the q / k / v product with 4-bit weights, every request's adapter beside it, rotary positions, the new rows into the paged
cache, attention over it, the output product and its adapters into the residual stream, the LM head, and a token for every request's
last row; first prompts, then single tokens, eagerly and as one replayed graph, and requests that end and make room for others.
Every operator is checked in its own file; here each stage is held against a plain statement in 64 bits of what the stage before it
left in memory, with the same bounds, so that a wrong hand-over shows as more than a rounding."""
import numpy as np
import pytest
import torch

from paper_2602_06412_b200 import binding as SL
from paper_2602_06412_b200 import inputs, sampler

from . import test_gemm_adapters as ad
from . import test_gemm_quantized as gq
from . import test_paged_plan as plan
from .test_paged_kv import DEV, Pool, _i32, _near, _want, quantise
from .test_rope import STEP, rotate
from .test_sample import choose

pytestmark = pytest.mark.gpu


class Server:
    """d_model 512, 4 query heads on 2 key heads of 128, four requests at a time on a pool of 30 pages of 16 tokens."""
    d, H, Hkv, dh, B, P, W, V, group, n_ad, rank = 512, 4, 2, 128, 4, 16, 10, 1000, 64, 3, 16

    def __init__(self, kind):
        self.kind, self.N = kind, self.P * self.W
        qkv = (self.H + 2 * self.Hkv) * self.dh
        self.Wqkv, self.wqkv = gq._weights(qkv, self.d, self.group, True, torch.bfloat16, seed=1)
        self.Wo, self.wo = gq._weights(self.d, self.H * self.dh, self.group, False, torch.float32, seed=2)
        self.head = (torch.randn(self.V, self.d, generator=torch.Generator().manual_seed(3)) * 0.1).to(torch.bfloat16)
        self.head_dev = self.head.to(DEV)
        self.ad_qkv, self.ad_o = ad._make(self.n_ad, self.rank, self.d, qkv, 4), ad._make(self.n_ad, self.rank, self.H * self.dh, self.d, 5)
        self.pool_qkv, self.pool_o = (SL.Adapters(*[t.to(DEV) for t in p]) for p in (self.ad_qkv, self.ad_o))
        self.which = [0, -1, 2, 0]
        self.which_dev = _i32(self.which)
        self.freq = 10000.0 ** (-np.arange(0, self.dh, 2) / self.dh)
        self.rope = SL.Rope(torch.tensor(self.freq, device=DEV))
        self.pool = Pool(kind, self.B, self.N, self.Hkv, self.dh, self.P, n_pages=self.B * self.W, spare=0)
        self.pool.table.fill_(-1)
        self.pool.dev_table.fill_(-1)
        self.n_pages = 30                                          # fewer than four whole requests need
        self.free = _i32(list(range(self.n_pages)))
        self.n_free, self.lens, self.status = _i32([self.n_pages]), _i32([0] * self.B), _i32([0])
        self.sets = dict(temperature=[0.8, 0.0, 1.2, 1.0], top_k=[50, 0, 0, 3], top_p=[0.9, 1.0, 0.95, 1.0], min_p=[0.0, 0.0, 0.05, 0.0])
        f = lambda n: torch.tensor(self.sets[n], dtype=torch.int32 if n == "top_k" else torch.float32, device=DEV)
        self.sampling = SL.Sampling(f("temperature"), f("top_k"), f("top_p"), f("min_p"))

    def buffers(self, M):
        z = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device=DEV)
        i = lambda n: z(n, t=torch.int32)
        return dict(x=z(M, self.d), qkv=z(M, self.wqkv.shape[0]), o=z(M, self.H * self.dh), res=z(M, self.d, t=torch.float32), last=z(self.B, self.d),
                    logits=z(self.B, self.V), new=i(self.B), offs=i(self.B + 1), idx=i(M), n=i(1), all=_i32([self.B]), u=z(self.B, t=torch.float32),
                    token=i(self.B), conf=z(self.B, t=torch.float32), kept=i(self.B), ws=z(SL.surelock_attention_paged_workspace_bytes(self.dh), t=torch.uint8),
                    projected=z(M, self.wqkv.shape[0]), turned=z(M, self.wqkv.shape[0]))

    def launch(self, t):
        """A step's calls on the current stream (and copies of what later calls overwrite, for the checks)."""
        SL.surelock_paged_extend(self.pool.dev_table, self.P, self.lens, t["new"], self.free, self.n_free, t["offs"], t["idx"], t["n"], dev_status=self.status)
        SL.surelock_gemm_quantized(t["x"], self.Wqkv, t["qkv"], t["n"], dev_status=self.status)
        t["projected"].copy_(t["qkv"])
        SL.surelock_gemm_adapters(t["x"], self.pool_qkv, self.which_dev, t["offs"], t["qkv"], self.status)
        t["turned"].copy_(t["qkv"])
        heads = t["qkv"].view(-1, self.H + 2 * self.Hkv, self.dh)
        q, k, v = heads[:, :self.H], heads[:, self.H:self.H + self.Hkv], heads[:, self.H + self.Hkv:]
        SL.surelock_rope(self.rope, q, k, t["idx"], t["n"], N=self.N, dev_status=self.status)
        SL.surelock_kv_scatter_paged(self.pool.cache, k, v, t["idx"], t["n"], self.N, self.status)
        SL.surelock_attention_paged(self.pool.cache, q, t["offs"], self.lens, t["o"].view(-1, self.H, self.dh), t["ws"], self.status)
        SL.surelock_gemm_quantized(t["o"], self.Wo, t["res"], t["n"], epilogue=1, dev_status=self.status)
        SL.surelock_gemm_adapters(t["o"], self.pool_o, self.which_dev, t["offs"], t["res"], self.status)
        t["last"].copy_(t["res"][(t["offs"][1:] - 1).clamp(min=0).long()])
        SL.surelock_gemm(t["last"], self.head_dev, t["logits"], t["all"])
        SL.surelock_sample(t["logits"], self.sampling, t["u"], t["all"], t["token"], t["conf"], t["kept"], dev_status=self.status)

    def fill(self, t, new, seed):
        g = torch.Generator().manual_seed(seed)
        for name in ("x", "res"):
            t[name].copy_(torch.randn(t[name].shape, generator=g))
        t["u"].copy_(torch.rand(self.B, generator=g))
        t["new"].copy_(_i32(new))
        before = [self.pool.dev_table.tolist(), self.lens.tolist(), self.free.tolist(), self.n_free.item(), t["res"].clone()]
        return before

    def check(self, t, new, before):
        table, lens, free, n_free, res0 = before
        np64 = lambda x: x.cpu().double().numpy()
        table, lens, top, offs, idx = plan.extend(table, self.P, lens, new, free, n_free, t["idx"].numel())
        M = offs[-1]
        assert (self.pool.dev_table.tolist(), self.lens.tolist(), self.n_free.item(), t["offs"].tolist(), t["idx"].tolist()[:M]) == (table, lens, top, offs, idx)
        self.pool.table.copy_(torch.tensor(table, dtype=torch.int32))
        x, raw, qkv, o = np64(t["x"][:M]), np64(t["projected"][:M]), np64(t["turned"][:M]), np64(t["o"][:M])
        assert np.all(np.abs(raw - x @ self.wqkv.T) <= gq._tol(x, self.wqkv, self.d, self.group) + 2.0 ** -8 * np.abs(x @ self.wqkv.T))
        want, tol = ad._want(t["x"][:M].cpu(), t["projected"][:M].cpu(), *self.ad_qkv, [self.rank] * self.n_ad, self.which, offs)
        # t has 17 bits: 2^-17 of sum |b| |t| scale, and |t| by its summands
        size, _ = ad._want(t["x"][:M].cpu().abs(), torch.zeros_like(t["projected"][:M]).cpu(), self.ad_qkv[0].abs(), self.ad_qkv[1].abs(), self.ad_qkv[2].abs(),
                           [self.rank] * self.n_ad, self.which, offs)
        assert np.all(np.abs(qkv - want) <= tol + 2.0 ** -17 * size + 2.0 ** -8 * np.abs(want))
        heads, got = qkv.reshape(M, -1, self.dh), np64(t["qkv"][:M]).reshape(M, -1, self.dh)
        pos = np.array(idx, dtype=np.int64) % self.N
        want, size = rotate(heads[:, :self.H + self.Hkv], pos, self.freq, False)
        assert np.all(np.abs(got[:, :self.H + self.Hkv] - want) <= 2.0 ** -21 * size + STEP[torch.bfloat16] * np.abs(want))
        assert np.array_equal(got[:, self.H + self.Hkv:], heads[:, self.H + self.Hkv:])
        for part, p, s in ((got[:, self.H:self.H + self.Hkv], self.pool.k, self.pool.ks), (got[:, self.H + self.Hkv:], self.pool.v, self.pool.vs)):
            for b in range(self.B):
                rows = range(offs[b], offs[b + 1])
                if len(rows):
                    place = [idx[r] % self.N for r in rows]
                    was = self.rows(p, b, lens[b])[place]
                    if s is None:
                        assert np.array_equal(was, part[rows])
                    else:
                        code, scale = quantise(part[rows], self.kind)
                        assert np.array_equal(was, code) and np.array_equal(self.rows(s, b, lens[b])[place].astype(np.float32), scale)
        self.pool.rows = self.rows
        want, A = _want(self.pool, got[:, :self.H], offs, lens, self.H // self.Hkv)
        _near(t["o"][:M].view(M, self.H, self.dh), want, A, self.kind)
        want, tol = ad._want(t["o"][:M].cpu(), torch.from_numpy(np64(res0[:M]) + o @ self.wo.T), *self.ad_o, [self.rank] * self.n_ad, self.which, offs)
        tol = tol + gq._tol(o, self.wo, self.H * self.dh, self.group) + 2.0 ** -23 * (np.abs(want) + np.abs(np64(res0[:M])))
        assert np.all(np.abs(np64(t["res"][:M]) - want) <= tol) and torch.equal(t["res"][M:], res0[M:])
        logits = np64(t["logits"])
        for b in range(self.B):
            s = {n: float(np.float32(v[b])) for n, v in self.sets.items()}
            token, conf, kept = choose(logits[b], t["u"][b].item(), s["temperature"], int(s["top_k"]), s["top_p"], s["min_p"])
            assert (t["token"][b].item(), t["kept"][b].item()) == (token, kept) and abs(t["conf"][b].item() - conf) <= 2.0 ** -19 * conf
        last, w = np64(t["last"]), self.head.double().numpy()
        assert np.array_equal(last, np64(t["res"][[max(0, n - 1) for n in offs[1:]]].to(torch.bfloat16)))
        assert np.all(np.abs(logits - last @ w.T) <= self.d * 2.0 ** -23 * (np.abs(last) @ np.abs(w).T) + 2.0 ** -8 * np.abs(last @ w.T))
        assert self.status.item() == 0
        return offs

    def rows(self, pool, b, n):
        """The first n rows of sequence b, on the CPU; a table has no pages behind its last token."""
        pages = [int(p) for p in self.pool.table[b, :-(-n // self.P)]]
        x = pool.view(torch.uint8) if pool.element_size() == 1 else pool
        x = torch.stack([x[p] for p in pages]).cpu()
        x = (x.view(pool.dtype) if pool.element_size() == 1 else x).to(torch.float32)
        return x.transpose(1, 2).reshape(-1, *([x.shape[1]] + list(x.shape[3:])))[:n].double().numpy()


@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float8_e4m3fn, torch.int8])
def test_prompts_tokens_and_requests_that_come_and_go(kind):
    s = Server(kind)
    t = s.buffers(200)
    new = (41, 100, 5, 17)
    before = s.fill(t, new, 1)
    s.launch(t)
    s.check(t, new, before)
    step = s.buffers(s.B)
    s.fill(step, (0, 0, 0, 0), 2)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.launch(step)
    for seed, new in enumerate([(1, 1, 1, 1), (1, 0, 1, 1), (0, 0, 0, 1)]):
        before = s.fill(step, new, 10 + seed)
        graph.replay()
        s.check(step, new, before)
    # the second ends, the third takes two tokens back; a new prompt in the second's place, and one for which no pages are left
    SL.surelock_paged_truncate(s.pool.dev_table, s.P, s.lens, _i32([999, 0, s.lens.tolist()[2] - 2, 999]), s.free, s.n_free, dev_status=s.status)
    new = (150 - s.lens.tolist()[0], 160, 1, 130)
    before = s.fill(t := s.buffers(500), new, 20)
    s.launch(t)
    offs = s.check(t, new, before)
    assert offs[4] == offs[3] and offs[2] > offs[1]
    for seed, new in enumerate([(1, 0, 1, 1), (1, 0, 1, 1)]):
        before = s.fill(step, new, 30 + seed)
        graph.replay()
        s.check(step, new, before)


def _decode(sampling, seed=0, steps=24):
    from tests.parity_util import to_dev
    cfg = inputs.model_shape("tiny")
    w = to_dev(inputs.make_weights(cfg, 9, dtype=torch.float32))
    B, N, n_prompt = 2, 128, 64
    ctx = SL.surelock_init(cfg, w, N, B)
    tokens, mask = (x.to(DEV) for x in inputs.make_tokens(B, N, n_prompt, cfg["vocab"], 5))
    r = sampler.run(ctx, tokens, mask, n_prompt, 32, steps, 1e-3, unmask_per_step=2, sampling=sampling)
    return tokens.cpu(), mask.cpu(), r


def test_the_decoding_loop_samples():
    greedy = _decode(None)
    zero = _decode(dict(temperature=0.0))
    assert torch.equal(greedy[0], zero[0]) and torch.equal(greedy[1], zero[1])          # temperature 0 is the argmax
    assert torch.equal(greedy[0], _decode(dict(top_k=1))[0])
    one, same, other = (_decode(dict(temperature=1.0, top_p=0.99, min_p=1e-4, seed=s)) for s in (1, 1, 2))
    assert torch.equal(one[0], same[0]) and not torch.equal(one[0], other[0]) and not torch.equal(one[0], greedy[0])
    for tokens, mask, r in (one, other):
        assert r["unmasked_per_step"] == greedy[2]["unmasked_per_step"] and int(tokens.min()) >= 0 and int(tokens.max()) < 2048
