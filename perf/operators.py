"""The operators for few active rows whose weights and caches are held in few bits, as measured cases.

  gemm       products of packed rows with 4-bit weights and group scales (store / += fp32 stream / SwiGLU)
  scatter    K/V rows written into a paged cache, quantised on the way
  gather     K/V rows read back from a paged cache
  attention  packed query rows against a paged cache (one new token per sequence up to some dozens of rows)

With `own` false, run() computes an operator in elementary torch operations; with `own` true it makes the call that a user
of the library makes.  exact() is the definition once more, in 64 bits, sequence by sequence or by blocks of outputs."""
import math

import torch

own = False

QMAX = {"e4m3": 448.0, "int8": 127.0}
CODE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8, "bf16": torch.bfloat16}
TYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
STORE, RESIDUAL, SWIGLU = 0, 1, 2


def listed():
    return [
        # output projection of one active row (LLaDA-8B shape): launch latency and 8 MB of weights
        dict(name="gemm 1 row 4096x4096", op="gemm", M=1, n_out=4096, K=4096, group=128, zeros=False, scale="bf16", epilogue=STORE),
        # gate and up projections with SwiGLU at a usual number of active rows late in a decoding run
        dict(name="gemm 23 rows gate/up", op="gemm", M=23, n_out=12288, K=4096, group=128, zeros=True, scale="bf16", epilogue=SWIGLU),
        # down projection into the residual stream, finer groups, fp32 scales, the most rows that count as few
        dict(name="gemm 128 rows down", op="gemm", M=128, n_out=4096, K=12288, group=64, zeros=True, scale="fp32", epilogue=RESIDUAL),
        # LM head over the whole vocabulary: the largest matrix
        dict(name="gemm 8 rows LM head", op="gemm", M=8, n_out=126464, K=4096, group=128, zeros=False, scale="bf16", epilogue=STORE),
        # a step with few active rows writes their K/V: latency
        dict(name="scatter int8 23 rows", op="scatter", kind="int8", B=1, N=512, rows=23, Hkv=32, dh=128, page=64, dtype="bf16"),
        # first step of a batch: every position of every sequence is written
        dict(name="scatter e4m3 8x1536 rows", op="scatter", kind="e4m3", B=8, N=1536, rows=1536, Hkv=32, dh=128, page=64, dtype="bf16"),
        # half of a batch's positions read back, e.g. into a contiguous cache
        dict(name="gather int8 8x768 rows", op="gather", kind="int8", B=8, N=1536, rows=768, Hkv=32, dh=128, page=64, dtype="bf16"),
        # small heads, odd counts, full-precision output
        dict(name="gather e4m3 3x77 rows", op="gather", kind="e4m3", B=3, N=301, rows=77, Hkv=4, dh=64, page=16, dtype="fp32"),
        # one sequence with a few active rows: the smallest attention of a step
        dict(name="attention int8 23 rows N512", op="attention", kind="int8", B=1, L=512, rows=23, ragged=False, Hkv=32, G=1, dh=128, page=64),
        # one new token for each of a ragged batch, grouped query heads
        dict(name="attention e4m3 1 row B32", op="attention", kind="e4m3", B=32, L=4099, rows=1, ragged=True, Hkv=8, G=4, dh=128, page=64),
        # long contexts
        dict(name="attention e4m3 1 row L16384", op="attention", kind="e4m3", B=4, L=16384, rows=1, ragged=False, Hkv=32, G=1, dh=128, page=128),
        # unquantised pages, small heads, more rows and ragged counts
        dict(name="attention bf16 33 rows dh64", op="attention", kind="bf16", B=5, L=1021, rows=33, ragged=True, Hkv=16, G=2, dh=64, page=16),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["gemm", "gemm", "scatter", "gather", "attention", "attention"])
    if op == "gemm":
        group = rng.choice([32, 64, 128])
        n_out, K = _log(rng, 48, 16000), group * _log(rng, 2, 14000 // group)
        return dict(op=op, M=_log(rng, 1, min(128, max(1, 3 * 10 ** 9 // (n_out * K)))), n_out=n_out, K=K, group=group,
                    zeros=rng.random() < 0.5, scale=rng.choice(["bf16", "fp32"]), epilogue=rng.choice([STORE, RESIDUAL, SWIGLU]))
    kind, Hkv, dh = rng.choice(["e4m3", "int8", "bf16"]), rng.choice([1, 2, 3, 8, 16, 32]), rng.choice([64, 128])
    page = rng.choice([16, 32, 64, 128, 256])
    if op in ("scatter", "gather"):
        N = _log(rng, 1, 4000)
        return dict(op=op, kind=kind, B=_log(rng, 1, 8) if N < 1536 else _log(rng, 1, 3), N=N, rows=_log(rng, 1, N), Hkv=Hkv, dh=dh, page=page,
                    dtype=rng.choice(["bf16", "fp32"]))
    G, B, rows = rng.choice([1, 2, 4, 7, 8]), _log(rng, 1, 64), rng.choice([1, 1, _log(rng, 2, 64)])
    # bounded by the cache and, for many rows, by the scores and the products
    most = min(32768, int(2.6e8 / (B * Hkv * dh * (2 if kind == "bf16" else 1))), int(1e8 / (B * Hkv * G * rows)), int(3.2e9 / (B * Hkv * G * rows * dh)))
    return dict(op=op, kind=kind, B=B, L=_log(rng, 1, max(1, most)), rows=rows, ragged=rng.random() < 0.7, Hkv=Hkv, G=G, dh=dh, page=page)


def _spread(most, B, ragged):
    """Sizes of B sequences: all `most`, or evenly from `most` down to half of it."""
    return [most - (b * (most // 2)) // max(1, B - 1) if ragged else most for b in range(B)]


def _counts(c):
    """Rows of each sequence of an attention case."""
    return [max(1, n) for n in _spread(c["rows"], c["B"], c["ragged"])]


def work(c):
    if c["op"] == "gemm":
        mats = 2 if c["epilogue"] == SWIGLU else 1
        ng = c["K"] // c["group"]
        weights = c["n_out"] * (c["K"] // 2 + ng * (2 if c["scale"] == "bf16" else 4) + (ng if c["zeros"] else 0))
        out = c["M"] * c["n_out"] * (8 if c["epilogue"] == RESIDUAL else 2)
        return {"bytes": mats * weights + 2 * c["M"] * c["K"] + out, "flops": 2.0 * mats * c["M"] * c["n_out"] * c["K"]}
    cached = c["dh"] * (2 if c["kind"] == "bf16" else 1) + (0 if c["kind"] == "bf16" else 4)   # bytes of one token's K (or V) of one head
    if c["op"] in ("scatter", "gather"):
        return {"bytes": 2 * c["B"] * c["rows"] * c["Hkv"] * (cached + c["dh"] * (2 if c["dtype"] == "bf16" else 4)), "flops": 0}
    lens, rows = _spread(c["L"], c["B"], c["ragged"]), _counts(c)
    H = c["Hkv"] * c["G"]
    return {"bytes": 2 * sum(lens) * c["Hkv"] * cached + 4 * sum(rows) * H * c["dh"],
            "flops": 4.0 * H * c["dh"] * sum(n * m for n, m in zip(lens, rows))}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _pages(g, c, tokens):
    """Page table of B sequences of `tokens` tokens over a pool in random order, with a few pages nobody uses."""
    per = (tokens + c["page"] - 1) // c["page"]
    n_pages = c["B"] * per + 3
    table = torch.randperm(n_pages, device="cuda", generator=g)[: c["B"] * per].to(torch.int32).reshape(c["B"], per)
    return n_pages, table.contiguous()


def _pool(g, c, n_pages):
    """A filled pool: codes as quantised normal values have them, with their scales; plain values for bf16."""
    shape = (n_pages, c["Hkv"], c["page"], c["dh"])
    x = _randn(g, *shape)
    if c["kind"] == "bf16":
        return x.to(torch.bfloat16), None
    q = QMAX[c["kind"]]
    x = (x * (q / 3.5)).clamp_(-q, q)
    x = x.round_().to(torch.int8) if c["kind"] == "int8" else x.to(torch.float8_e4m3fn)
    return x, (torch.rand(shape[:3], device="cuda", generator=g) + 0.5) * (3.5 / q)


def _cache(g, c, tokens, filled):
    n_pages, table = _pages(g, c, tokens)
    s = {"table": table}
    for name in ("k", "v"):
        if filled:
            s["pool_" + name], s["scale_" + name] = _pool(g, c, n_pages)
        else:
            s["pool_" + name] = torch.zeros((n_pages, c["Hkv"], c["page"], c["dh"]), device="cuda").to(CODE[c["kind"]])
            s["scale_" + name] = None if c["kind"] == "bf16" else torch.zeros((n_pages, c["Hkv"], c["page"]), device="cuda")
    return s


def _count(n):
    return torch.tensor([n], dtype=torch.int32, device="cuda")


def _positions(g, c):
    """`rows` positions of each of B sequences of N, ascending: flat b * N + i, as the active rows of a step come."""
    order = torch.rand((c["B"], c["N"]), device="cuda", generator=g).argsort(1)[:, : c["rows"]].sort(1).values
    return (order + torch.arange(c["B"], device="cuda")[:, None] * c["N"]).reshape(-1).to(torch.int32)


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = {"c": c}
    if c["op"] == "gemm":
        n, K, ng = c["n_out"], c["K"], c["K"] // c["group"]
        s["A"] = _randn(g, c["M"], K).to(torch.bfloat16)
        for i in range(2 if c["epilogue"] == SWIGLU else 1):
            codes = torch.randint(0, 256, (n, K // 2), device="cuda", generator=g, dtype=torch.uint8)
            scale = ((torch.rand((n, ng), device="cuda", generator=g) + 0.5) * 0.004).to(TYPE[c["scale"]])
            zero = torch.randint(5, 11, (n, ng), device="cuda", generator=g, dtype=torch.uint8) if c["zeros"] else None
            s["W%d" % i] = (codes, scale, zero)
        s["C"] = _randn(g, c["M"], n) if c["epilogue"] == RESIDUAL else torch.empty((c["M"], n), dtype=torch.bfloat16, device="cuda")
        s["n"] = _count(c["M"])
        return s
    if c["op"] == "attention":
        lens, rows = _spread(c["L"], c["B"], c["ragged"]), _counts(c)
        at = torch.randperm(c["B"], device="cuda", generator=g)
        s.update(_cache(g, c, c["L"], True))
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")[at].contiguous()
        counts = torch.tensor(rows, dtype=torch.int32, device="cuda")[at]
        s["offsets"] = torch.cat([torch.zeros_like(counts[:1]), counts.cumsum(0)]).to(torch.int32)
        s["q"] = (_randn(g, sum(rows), c["Hkv"] * c["G"], c["dh"]) * 1.5).to(torch.bfloat16)
        s["o"] = torch.empty_like(s["q"])
        return s
    s.update(_cache(g, c, c["N"], c["op"] == "gather"))
    s["idx"] = _positions(g, c)
    s["n"] = _count(s["idx"].numel())
    shape = (s["idx"].numel(), c["Hkv"], c["dh"])
    if c["op"] == "scatter":
        # heads of different magnitude, as keys and values have them
        size = torch.exp(_randn(g, 1, c["Hkv"], 1))
        s["k"], s["v"] = ((_randn(g, *shape) * size).to(TYPE[c["dtype"]]) for _ in range(2))
    else:
        s["k"], s["v"] = (torch.empty(shape, dtype=TYPE[c["dtype"]], device="cuda") for _ in range(2))
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------------
def _weights(W, group):
    codes, scale, zero = W
    u = torch.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1, group).float()
    return ((u - (8.0 if zero is None else zero.float()[:, :, None])) * scale.float()[:, :, None]).reshape(codes.shape[0], -1)


def _slots(s, idx):
    """Page and place in the page of flat positions."""
    c = s["c"]
    b, i = idx.long() // c["N"], idx.long() % c["N"]
    return s["table"][b, i // c["page"]].long(), i % c["page"]


def _quantised(x, kind):
    """(codes, scales) of x [rows][heads][dh]: scale = largest magnitude / largest code in 32 bits, codes rounded to nearest even
    from the quotient in 64 bits (32 would put some next to a border on the wrong side)."""
    scale = (x.abs().amax(2).double() / QMAX[kind]).float()
    q = x.double() / torch.where(scale == 0, torch.ones_like(scale), scale).double()[:, :, None]
    q = q.clamp(-QMAX[kind], QMAX[kind])
    if kind == "int8":
        return q.round().to(torch.int8), scale
    step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)   # three mantissa bits; below 2^-6 the spacing stays
    return ((q / step).round() * step).float().to(torch.float8_e4m3fn), scale


def _put(pool, at, values):
    """pool[page, :, place] = values; one-byte pools go by their bytes."""
    if pool.element_size() == 1:
        pool, values = pool.view(torch.uint8), values.contiguous().view(torch.uint8)
    pool[at[0], :, at[1]] = values


def _plain(s):
    c = s["c"]
    if c["op"] == "gemm":
        A = s["A"].float()
        y = A @ _weights(s["W0"], c["group"]).T
        if c["epilogue"] == RESIDUAL:
            s["C"] += y
            return s["C"]
        if c["epilogue"] == SWIGLU:
            y = y / (1 + torch.exp(-y)) * (A @ _weights(s["W1"], c["group"]).T)
        return y.to(torch.bfloat16)
    if c["op"] == "scatter":
        at = _slots(s, s["idx"])
        out = {}
        for name in ("k", "v"):
            codes, scale = (s[name].to(torch.bfloat16), None) if c["kind"] == "bf16" else _quantised(s[name].float(), c["kind"])
            _put(s["pool_" + name], at, codes)
            if scale is not None:
                _put(s["scale_" + name], at, scale)
            out[name], out[name + "_scale"] = s["pool_" + name], s["scale_" + name]
        return out
    if c["op"] == "gather":
        page, place = _slots(s, s["idx"])
        out = {}
        for name in ("k", "v"):
            x = s["pool_" + name].view(torch.uint8 if c["kind"] != "bf16" else torch.bfloat16)[page, :, place].contiguous()
            x = x.view(CODE[c["kind"]]).float()
            if c["kind"] != "bf16":
                x = x * s["scale_" + name][page, :, place][:, :, None]
            out[name] = x.to(TYPE[c["dtype"]])
        return out
    # attention: sequences padded to the longest, rows to the most
    B, Hkv, G, dh, L = c["B"], c["Hkv"], c["G"], c["dh"], c["L"]
    kv = []
    for name in ("k", "v"):
        x = s["pool_" + name].view(torch.uint8 if c["kind"] != "bf16" else torch.bfloat16)[s["table"].long()].view(CODE[c["kind"]]).float()
        if c["kind"] != "bf16":
            x = x * s["scale_" + name][s["table"].long()][..., None]
        kv.append(x.transpose(1, 2).reshape(B, Hkv, -1, dh)[:, :, :L])   # [B][pages][Hkv][page][dh] -> [B][Hkv][token][dh]
    offs = s["offsets"].long()
    row = torch.arange(s["q"].shape[0], device="cuda")
    b = (row[:, None] >= offs[None, 1:]).sum(1)
    r = row - offs[b]
    q = torch.zeros((B, c["rows"], Hkv, G, dh), device="cuda")
    q[b, r] = s["q"].float().reshape(-1, Hkv, G, dh)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, dh)
    p = q @ kv[0].transpose(2, 3) / math.sqrt(dh)
    inside = torch.arange(L, device="cuda")[None, :] < s["lens"][:, None]
    p = torch.where(inside[:, None, None, :], p, -math.inf)
    p = torch.exp(p - p.amax(3, keepdim=True))
    o = (p @ kv[1]) / p.sum(3, keepdim=True)
    o = o.reshape(B, Hkv, c["rows"], G, dh).permute(0, 2, 1, 3, 4)[b, r]
    return o.reshape(s["q"].shape).to(torch.bfloat16)


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_2602_06412_b200 import binding as SL
    c = s["c"]
    if c["op"] == "gemm":
        SL.surelock_gemm_quantized(s["A"], s["W0"], s["C"], s["n"], epilogue=c["epilogue"], W2=s.get("W1"))
        return s["C"]
    if "cache" not in s:   # the handle of the pool, and the workspace, that a program keeps
        s["cache"] = SL.PagedKV(s["pool_k"], s["pool_v"], s["table"], s["scale_k"], s["scale_v"])
        if c["op"] == "attention":
            s["workspace"] = torch.empty(SL.surelock_attention_paged_workspace_bytes(c["dh"]), dtype=torch.uint8, device="cuda")
    if c["op"] == "scatter":
        SL.surelock_kv_scatter_paged(s["cache"], s["k"], s["v"], s["idx"], s["n"], c["N"])
        return {"k": s["pool_k"], "k_scale": s["scale_k"], "v": s["pool_v"], "v_scale": s["scale_v"]}
    if c["op"] == "gather":
        SL.surelock_kv_gather_paged(s["cache"], s["idx"], s["n"], c["N"], s["k"], s["v"])
        return {"k": s["k"], "v": s["v"]}
    SL.surelock_attention_paged(s["cache"], s["q"], s["offsets"], s["lens"], s["o"], s["workspace"])
    return s["o"]


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def _exact_gemm(s):
    c = s["c"]
    A = s["A"].double()

    def product(W):
        codes, scale, zero = W
        out = []
        for lo in range(0, c["n_out"], 8192):   # 8192 output features at a time
            byte = codes[lo: lo + 8192].to(torch.int16)
            w = torch.empty((byte.shape[0], c["K"]), dtype=torch.float64, device="cuda")
            w[:, 0::2] = (byte % 16).double()
            w[:, 1::2] = (byte // 16).double()
            w = w.view(byte.shape[0], -1, c["group"])
            w -= 8 if zero is None else zero[lo: lo + 8192].double().unsqueeze(2)
            w *= scale[lo: lo + 8192].double().unsqueeze(2)
            out.append(torch.einsum("mk,nk->mn", A, w.view(byte.shape[0], -1)))
        return torch.cat(out, 1)

    y = product(s["W0"])
    if c["epilogue"] == RESIDUAL:
        return s["C"].double() + y
    if c["epilogue"] == SWIGLU:
        return y * torch.sigmoid(y) * product(s["W1"])
    return y


def _grid(q, kind):
    """The representable value of `kind` next to each q, ties to the even one."""
    if kind == "int8":
        return torch.round(q).clamp(-127, 127)
    values = torch.tensor([(m / 8.0) * 2.0 ** -6 for m in range(8)] + [(1 + m / 8.0) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1],
                          dtype=torch.float64, device="cuda")
    mid = (values[1:] + values[:-1]) / 2
    a = q.abs()
    above, upto = torch.bucketize(a, mid), torch.bucketize(a, mid, right=True)   # they differ on a midpoint only
    code = torch.where(above % 2 == 0, above, upto)
    return values[code] * torch.sign(q)


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "gemm":
        return _exact_gemm(s)
    if c["op"] == "attention":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
        offs, lens = s["offsets"].tolist(), s["lens"].tolist()
        for b in range(c["B"]):
            n, pages = lens[b], s["table"][b].long()
            for h in range(c["Hkv"]):
                k, v = (s["pool_" + name][:, h][pages] if c["kind"] == "bf16" else s["pool_" + name].view(torch.uint8)[:, h][pages].view(CODE[c["kind"]])
                        for name in ("k", "v"))
                k, v = k.double().reshape(-1, c["dh"])[:n], v.double().reshape(-1, c["dh"])[:n]
                if c["kind"] != "bf16":
                    k *= s["scale_k"][:, h][pages].double().reshape(-1, 1)[:n]
                    v *= s["scale_v"][:, h][pages].double().reshape(-1, 1)[:n]
                heads = slice(h * c["G"], (h + 1) * c["G"])
                x = torch.einsum("rgd,nd->rgn", s["q"][offs[b]: offs[b + 1], heads].double(), k) / math.sqrt(c["dh"])
                out[offs[b]: offs[b + 1], heads] = torch.einsum("rgn,nd->rgd", torch.softmax(x, 2), v)
        return out
    flat = s["idx"].tolist()
    table = s["table"].tolist()
    page = torch.tensor([table[f // c["N"]][(f % c["N"]) // c["page"]] for f in flat], device="cuda")
    place = torch.tensor([(f % c["N"]) % c["page"] for f in flat], device="cuda")
    out = {}
    for name in ("k", "v"):
        pool, scale = s["pool_" + name], s["scale_" + name]
        if c["op"] == "gather":
            x = pool.float()[page, :, place].double()
            out[name] = x if scale is None else x * scale[page, :, place].double().unsqueeze(2)
            continue
        x = s[name].double()
        new, new_scale = torch.zeros(pool.shape, dtype=torch.float64, device="cuda"), None
        if scale is None:
            new[page, :, place] = x
        else:
            top = x.abs().amax(2) / QMAX[c["kind"]]
            new_scale = torch.zeros(scale.shape, dtype=torch.float64, device="cuda")
            new_scale[page, :, place] = top
            stored = top.float().double()   # the scale is kept in 32 bits, and the codes are those of the kept one
            new[page, :, place] = _grid(x / torch.where(stored == 0, torch.ones_like(stored), stored).unsqueeze(2), c["kind"])
        out[name], out[name + "_scale"] = new.to(torch.int8) if c["kind"] == "int8" else new, new_scale
    return out
