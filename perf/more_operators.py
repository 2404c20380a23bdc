"""The operators that take a served batch on the paged cache from request lengths to tokens, as measured cases.

  extend    pages, row offsets and flat positions for the new tokens of every sequence
  truncate  sequences cut to given lengths, their pages returned to the free list
  rope      rotary positions on packed q and k rows
  adapters  low-rank adapters of many requests added to a shared projection
  sample    a token per row of logits from one given uniform number: temperature, top-k, top-p, min-p

With `own` false, run() computes an operator in elementary torch operations; with `own` true it makes the call that a user
of the library makes.  exact() is the definition once more, in 64 bits, sequence by sequence or row by row."""
import math

import torch

own = False

TYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # a decoding step of 32 requests: one token each, a new page now and then; latency
        dict(name="extend 32 x 1 token", op="extend", B=32, have=1500, new=1, page=64, width=64, tight=False),
        # a batch of prompts, ragged up to one benchmark sequence, more than the pool has pages for
        dict(name="extend 8 prompts tight", op="extend", B=8, have=1, new=1536, page=16, width=128, tight=True),
        # requests that take back the tokens of their last step, or end
        dict(name="truncate 32", op="truncate", B=32, have=1500, page=64, width=64),
        # most requests of a large batch end at once
        dict(name="truncate 900", op="truncate", B=900, have=2000, page=16, width=128),
        # one new token for each of 32 requests, far into long contexts, grouped heads
        dict(name="rope 32 rows far", op="rope", M=32, H=32, Hkv=8, dh=128, rot=128, interleaved=False, dtype="bf16", far=1000000, factor=8.0, theta=500000.0),
        # every row of a benchmark batch, 8 sequences of 1536
        dict(name="rope 8x1536 rows", op="rope", M=12288, H=32, Hkv=32, dh=128, rot=128, interleaved=False, dtype="bf16", far=1536, factor=1.0, theta=500000.0),
        # one request's token at the output projection (LLaDA-8B shape): latency
        dict(name="adapters 1 row", op="adapters", B=1, rows=1, ragged=False, n_ad=4, rank=16, K=4096, n_out=4096, out="bf16"),
        # 64 requests, one token each, adapters of several ranks, the gate projection
        dict(name="adapters 64 x 1 row", op="adapters", B=64, rows=1, ragged=False, n_ad=48, rank=64, K=4096, n_out=12288, out="bf16"),
        # a ragged batch of prompts through the output projection into the residual stream
        dict(name="adapters 8x1536 rows", op="adapters", B=8, rows=1536, ragged=True, n_ad=8, rank=32, K=4096, n_out=4096, out="fp32"),
        # one request with the usual settings of a chat, over the whole vocabulary: latency
        dict(name="sample 1 row", op="sample", M=1, V=126464, dtype="bf16", sets=1, temperature=0.8, top_k=50, top_p=0.95, min_p=0.0),
        # 33 requests with settings of their own, odd vocabulary, fp32 logits
        dict(name="sample 33 rows fp32", op="sample", M=33, V=32003, dtype="fp32", sets=33, temperature=1.0, top_k=200, top_p=0.9, min_p=0.02),
        # every position of a benchmark sequence samples from its posterior
        dict(name="sample 1536 rows", op="sample", M=1536, V=126464, dtype="bf16", sets=1, temperature=1.0, top_k=0, top_p=0.95, min_p=0.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["extend", "truncate", "rope", "rope", "adapters", "adapters", "sample", "sample", "sample"])
    if op in ("extend", "truncate"):
        page, B = rng.choice([16, 32, 64, 128, 256]), _log(rng, 1, 1024)
        width = _log(rng, 1, max(1, min(4096 // page * 4, 2 ** 19 // B)))
        have = rng.randint(0, page * width)
        if op == "truncate":
            return dict(op=op, B=B, have=have, page=page, width=width)
        return dict(op=op, B=B, have=have, new=rng.choice([1, 1, _log(rng, 2, max(2, min(page * width, 2 ** 18 // B)))]), page=page, width=width,
                    tight=rng.random() < 0.4)
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op == "rope":
        dh = rng.choice([64, 96, 128, 256])
        Hkv = rng.choice([1, 2, 8, 16, 32])
        H = Hkv * rng.choice([1, 2, 4, 7]) if Hkv <= 8 else 32
        return dict(op=op, M=_log(rng, 1, min(12288, 10 ** 8 // ((H + Hkv) * dh * (1 if dtype == "bf16" else 2)))), H=H, Hkv=Hkv, dh=dh,
                    rot=rng.choice([dh, dh, dh // 2, dh // 4]), interleaved=rng.random() < 0.4, dtype=dtype, far=_log(rng, 300, 2 ** 31 - 2),
                    factor=rng.choice([1.0, 1.0, 4.0, 32.0]), theta=rng.choice([10000.0, 500000.0]))
    if op == "adapters":
        K, n_out, rank = 8 * _log(rng, 8, 1536), _log(rng, 48, 12288), rng.choice([8, 16, 16, 32, 64, 128])
        B = _log(rng, 1, 100)
        most = min(1536, 4 * 10 ** 7 // (B * K), 4 * 10 ** 7 // (B * n_out), 10 ** 9 * 3 // (B * rank * (K + n_out)))
        rows = rng.choice([1, 1, _log(rng, 2, max(2, most))])
        return dict(op=op, B=B, rows=rows, ragged=rng.random() < 0.6, n_ad=_log(rng, 1, max(1, min(100, 2 * 10 ** 8 // (rank * (K + n_out)), 10 ** 7 // (B * rows * rank)))),
                    rank=rank, K=K, n_out=n_out, out=dtype)
    V = rng.choice([126464, 32000, 50257, _log(rng, 2, 200000)])
    M = _log(rng, 1, min(1536, (2 * 10 ** 8 if dtype == "bf16" else 10 ** 7) // V))
    return dict(op=op, M=M, V=V, dtype=dtype, sets=rng.choice([1, M]), temperature=rng.choice([0.0, 0.3, 0.7, 1.0, 1.0, 1.7]),
                top_k=rng.choice([0, 0, 1, 50, _log(rng, 1, V)]), top_p=rng.choice([1.0, 1.0, 0.5, 0.95, 0.999]), min_p=rng.choice([0.0, 0.0, 0.05, 0.3]))


def _ceil(a, b):
    return (a + b - 1) // b


def _rows_of(c):
    """Rows of each sequence of an adapters case: all `rows`, or evenly from `rows` down to half of it."""
    return [max(1, c["rows"] - (b * (c["rows"] // 2)) // max(1, c["B"] - 1)) if c["ragged"] else c["rows"] for b in range(c["B"])]


def work(c):
    if c["op"] == "extend":
        rows = c["B"] * (c["new"] if c["new"] == 1 else c["new"] * 0.75)
        return {"bytes": 16 * c["B"] + 4 * rows + 8 * rows / c["page"], "flops": 0}
    if c["op"] == "truncate":
        return {"bytes": 12 * c["B"] + 8 * c["B"] * c["have"] * 0.4 / c["page"], "flops": 0}
    size = 2 if c.get("dtype", c.get("out")) == "bf16" else 4
    if c["op"] == "rope":
        return {"bytes": 2.0 * size * c["M"] * (c["H"] + c["Hkv"]) * c["dh"] + 4 * c["M"], "flops": 3.0 * c["M"] * (c["H"] + c["Hkv"]) * c["rot"]}
    if c["op"] == "adapters":
        M, used = sum(_rows_of(c)), min(c["n_ad"], c["B"])
        return {"bytes": 2.0 * M * c["K"] + 2.0 * size * M * c["n_out"] + 2.0 * 0.7 * used * c["rank"] * (c["K"] + c["n_out"]),
                "flops": 2.0 * 0.7 * M * c["rank"] * (c["K"] + c["n_out"])}
    return {"bytes": size * c["M"] * c["V"] + 16 * c["M"], "flops": 2.0 * c["M"] * c["V"]}


def _randint(g, lo, hi, *shape):
    """Whole numbers from lo to hi, both included."""
    return torch.randint(lo, hi + 1, shape, device="cuda", generator=g)


def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _rand(g, *shape):
    return torch.rand(shape, device="cuda", generator=g)


def _int(x):
    return x.to(torch.int32).contiguous()


def _prepare_pages(c, g):
    """A pool whose pages lie in random order on the tables of B sequences or on the free list."""
    B, P, W = c["B"], c["page"], c["width"]
    lens = _randint(g, c["have"] // 2, c["have"], B)
    s = {"page": P}
    used, n_pages = _ceil(lens, P), B * W + 5
    mine = int(used.sum())
    if c["op"] == "extend":
        new = torch.ones_like(lens) if c["new"] == 1 else _randint(g, c["new"] // 2, c["new"], B)
        need = int((_ceil(lens + new, P) - used).sum())
        spare = min(n_pages - mine, need // 2 if c["tight"] else need + 3)    # the other pages are somebody else's
        s["new"], s["rows"] = _int(new), B * c["new"]
    else:
        spare = n_pages - mine
        kind = _randint(g, 0, 3, B)    # ended, cut back a little, cut to anything, left alone
        keep = torch.where(kind == 0, 0, torch.where(kind == 1, lens - 3, torch.where(kind == 2, (lens * _rand(g, B)).long(), lens + 7)))
        s["keep"] = _int(keep.clamp(min=0))
    order = torch.randperm(n_pages, device="cuda", generator=g)
    table, free = torch.full((B, W), -1, device="cuda"), torch.full((n_pages,), -1, device="cuda")
    table[torch.arange(W, device="cuda") < used[:, None]] = order[:mine]
    free[:spare] = order[mine: mine + spare]
    s.update(table=_int(table), lens=_int(lens), free=_int(free), n_free=_int(torch.tensor([spare], device="cuda")))
    s["lens_out"], s["n_free_out"] = torch.zeros_like(s["lens"]), torch.zeros_like(s["n_free"])
    if c["op"] == "extend":
        s["offsets"] = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        s["idx"] = torch.zeros(s["rows"], dtype=torch.int32, device="cuda")
        s["n"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return s


def prepare(case, seed):
    c, g = case, torch.Generator(device="cuda").manual_seed(int(seed))
    s = {"c": c}
    if c["op"] in ("extend", "truncate"):
        s.update(_prepare_pages(c, g))
    elif c["op"] == "rope":
        half = torch.arange(0, c["rot"], 2, dtype=torch.float64, device="cuda")
        s["freq"] = torch.exp(half * (-math.log(c["theta"]) / c["rot"])) / c["factor"]
        s["pos"] = _int(_randint(g, 0, c["far"], c["M"]))
        s["n"] = _int(torch.tensor([c["M"]], device="cuda"))
        for name, heads in (("q", c["H"]), ("k", c["Hkv"])):
            s[name] = _randn(g, c["M"], heads, c["dh"]).to(TYPE[c["dtype"]])
            s[name + "_out"] = torch.empty_like(s[name])
    elif c["op"] == "adapters":
        rows = _rows_of(c)
        M = sum(rows)
        s["x"] = _randn(g, M, c["K"]).to(torch.bfloat16)
        s["a"] = (_randn(g, c["n_ad"], c["rank"], c["K"]) * c["K"] ** -0.5).to(torch.bfloat16)
        s["b"] = (_randn(g, c["n_ad"], c["n_out"], c["rank"]) * 0.1).to(torch.bfloat16)
        s["scale"] = 0.5 + _rand(g, c["n_ad"]) * 1.5
        # whole ranks mostly, and some lower ones in the same pool
        s["ranks"] = _int(torch.where(_rand(g, c["n_ad"]) < 0.5, c["rank"], _randint(g, 1, c["rank"], c["n_ad"])))
        which = _randint(g, 0, c["n_ad"] - 1, c["B"])
        if c["B"] > 3:
            which = torch.where(_rand(g, c["B"]) < 0.1, -1, which)    # a request without an adapter
        s["which"] = _int(which)
        counts = torch.tensor(rows, device="cuda")
        s["offsets"] = _int(torch.cat([torch.zeros_like(counts[:1]), counts.cumsum(0)]))
        s["y"] = _randn(g, M, c["n_out"]).to(TYPE[c["out"]])
    else:
        M, V, n = c["M"], c["V"], c["sets"]
        x = _randn(g, M, V) * 3
        row = torch.arange(M, device="cuda")
        x[row, _randint(g, 0, V - 1, M)] += 15.0 * (row % 4 == 1)               # a confident row
        out = (_rand(g, M, V) < 0.3) & ((row % 8 == 5) & (V > 8))[:, None]       # tokens that a grammar forbids
        s["logits"] = x.masked_fill_(out, -math.inf).to(TYPE[c["dtype"]])
        s["u"] = _rand(g, M)
        own_sets = n > 1
        s["temperature"] = c["temperature"] * (0.5 + _rand(g, n)) * (_rand(g, n) < 0.85) if own_sets else torch.full((1,), c["temperature"], device="cuda")
        s["top_k"] = _int(_randint(g, 0, c["top_k"], n)) if own_sets else _int(torch.tensor([c["top_k"]], device="cuda"))
        s["top_p"] = 1 - (1 - c["top_p"]) * 2 * _rand(g, n) if own_sets else torch.full((1,), c["top_p"], device="cuda")
        s["min_p"] = c["min_p"] * 2 * _rand(g, n) if own_sets else torch.full((1,), c["min_p"], device="cuda")
        s["n"] = _int(torch.tensor([M], device="cuda"))
        s["token"], s["kept"] = (torch.zeros(M, dtype=torch.int32, device="cuda") for _ in range(2))
        s["conf"] = torch.zeros(M, device="cuda")
    return s


# ---- plain forms -------------------------------------------------------------------------------------------------------
def _plain_extend(s):
    c = s["c"]
    P, W, N = c["page"], c["width"], c["page"] * c["width"]
    lens, new, n_free = s["lens"].long(), s["new"].long(), s["n_free"].long()
    have = _ceil(lens, P)
    need = _ceil(lens + new, P) - have
    fits = lens + new <= N
    ok = fits & ((need == 0) | (torch.where(fits, need, 0).cumsum(0) <= n_free)) & (torch.where(fits, new, 0).cumsum(0) <= s["rows"])
    need, new = torch.where(ok, need, 0), torch.where(ok, new, 0)
    first = need.cumsum(0) - need
    col = torch.arange(W, device="cuda")
    fresh = (col >= have[:, None]) & (col < (have + need)[:, None])
    at = (n_free - 1 - first[:, None] - col + have[:, None]).clamp(0, s["free"].numel() - 1)
    table = torch.where(fresh, s["free"].long()[at], s["table"].long())
    offsets = torch.cat([torch.zeros_like(new[:1]), new.cumsum(0)])
    r = torch.arange(s["rows"], device="cuda")
    b = torch.searchsorted(offsets[1:], r, right=True).clamp(max=c["B"] - 1)
    idx = torch.where(r < offsets[-1], b * N + lens[b] + r - offsets[b], s["idx"].long())
    out = dict(table=table, lens=lens + new, n_free=n_free - need.sum(), offsets=offsets, idx=idx, n=offsets[-1:])
    return {k: v.to(torch.int32) for k, v in out.items()}


def _plain_truncate(s):
    c = s["c"]
    P = c["page"]
    lens, n_free, table = s["lens"].long(), s["n_free"].long(), s["table"].long()
    keep = torch.minimum(s["keep"].long(), lens)
    first, last = _ceil(keep, P), _ceil(lens, P)
    count = last - first
    col = torch.arange(c["width"], device="cuda")
    gone = (col >= first[:, None]) & (col < last[:, None])
    to = torch.where(gone, n_free + (count.cumsum(0) - count - first)[:, None] + col, s["free"].numel())
    free = torch.cat([s["free"].long(), s["free"].long()[:1]])
    free[to.reshape(-1)] = table.reshape(-1)
    return dict(free=free[:-1].to(torch.int32), lens=keep.to(torch.int32), n_free=(n_free + count.sum()).to(torch.int32))


def _plain_rope(s):
    c = s["c"]
    angle = s["pos"].double()[:, None] * s["freq"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    out = {}
    for name in ("q", "k"):
        x = s[name].float()
        part, rest = x[..., : c["rot"]], x[..., c["rot"]:]
        if c["interleaved"]:
            a, b = part[..., 0::2], part[..., 1::2]
            part = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = part[..., : c["rot"] // 2], part[..., c["rot"] // 2:]
            part = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        out[name] = torch.cat([part, rest], -1).to(s[name].dtype)
    return out


def _plain_adapters(s):
    c = s["c"]
    M = s["x"].shape[0]
    seq = torch.searchsorted(s["offsets"].long()[1:], torch.arange(M, device="cuda"), right=True)
    which = s["which"].long()[seq]
    # all adapters at once, and of every row the columns of its own
    t = (s["x"].float() @ s["a"].float().reshape(-1, c["K"]).T).reshape(M, c["n_ad"], c["rank"])
    mine = (which[:, None] == torch.arange(c["n_ad"], device="cuda"))[:, :, None] & \
        (torch.arange(c["rank"], device="cuda") < s["ranks"].long()[:, None])[None]
    t = torch.where(mine, t * s["scale"][None, :, None], 0.0)
    y = t.reshape(M, -1) @ s["b"].float().transpose(1, 2).reshape(-1, c["n_out"])
    return s["y"].copy_(s["y"].float() + y)


def _plain_sample(s):
    x, order = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    V = x.shape[1]
    z = x.double() - x[:, :1].double()
    T, k, p, m = (s[name][:, None].expand(x.shape[0], 1) for name in ("temperature", "top_k", "top_p", "min_p"))
    greedy = T == 0
    w = torch.exp(z / torch.where(greedy, 1.0, T).double())
    cum = w.cumsum(1)
    finite = (x > -math.inf).sum(1, keepdim=True)
    n = torch.where(k > 0, torch.minimum(k.long(), finite), finite)
    total = cum.gather(1, n - 1)
    n = torch.where(p < 1, torch.minimum(n, (cum < p.double() * total).sum(1, keepdim=True) + 1), n)
    n = torch.minimum(n, (w >= m.double()).sum(1, keepdim=True).clamp(min=1))
    n = torch.where(greedy, 1, n)
    target = s["u"].double()[:, None] * cum.gather(1, n - 1)
    j = torch.minimum((cum <= target).sum(1, keepdim=True), n - 1).clamp(max=V - 1)
    conf = torch.exp(z.gather(1, j)) / torch.exp(z).sum(1, keepdim=True)
    return dict(token=order.gather(1, j)[:, 0].to(torch.int32), conf=conf[:, 0].float(), kept=n[:, 0].to(torch.int32))


def run(state):
    s = state
    c = s["c"]
    if not own:
        return {"extend": _plain_extend, "truncate": _plain_truncate, "rope": _plain_rope, "adapters": _plain_adapters, "sample": _plain_sample}[c["op"]](s)
    from paper_2602_06412_b200 import binding as SL
    if c["op"] == "extend":
        SL.surelock_paged_extend(s["table"], c["page"], s["lens"], s["new"], s["free"], s["n_free"], s["offsets"], s["idx"], s["n"],
                                 seq_lens_out=s["lens_out"], n_free_out=s["n_free_out"])
        return dict(table=s["table"], lens=s["lens_out"], n_free=s["n_free_out"], offsets=s["offsets"], idx=s["idx"], n=s["n"])
    if c["op"] == "truncate":
        SL.surelock_paged_truncate(s["table"], c["page"], s["lens"], s["keep"], s["free"], s["n_free"], seq_lens_out=s["lens_out"],
                                   n_free_out=s["n_free_out"])
        return dict(free=s["free"], lens=s["lens_out"], n_free=s["n_free_out"])
    if c["op"] == "rope":
        if "rope" not in s:    # the handle of the frequencies that a program keeps
            s["rope"] = SL.Rope(s["freq"], interleaved=c["interleaved"])
        SL.surelock_rope(s["rope"], s["q"], s["k"], s["pos"], s["n"], q_out=s["q_out"], k_out=s["k_out"])
        return dict(q=s["q_out"], k=s["k_out"])
    if c["op"] == "adapters":
        if "adapters" not in s:    # the handle of the pool that a program keeps
            s["adapters"] = SL.Adapters(s["a"], s["b"], s["scale"], s["ranks"])
        SL.surelock_gemm_adapters(s["x"], s["adapters"], s["which"], s["offsets"], s["y"])
        return s["y"]
    if "sampling" not in s:    # the settings of the requests that a program keeps
        s["sampling"] = SL.Sampling(s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    SL.surelock_sample(s["logits"], s["sampling"], s["u"], s["n"], s["token"], s["conf"], s["kept"])
    return dict(token=s["token"], conf=s["conf"], kept=s["kept"])


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def _exact_sample(s):
    token, conf, kept = [], [], []
    sets = {name: s[name].cpu() for name in ("temperature", "top_k", "top_p", "min_p")}
    for r in range(s["logits"].shape[0]):
        T, k, p, m = (float(sets[name][r % sets[name].numel()]) for name in ("temperature", "top_k", "top_p", "min_p"))
        v = s["logits"][r].double()
        v = torch.where(v == -math.inf, v, v - v.max())
        order = torch.argsort(v, descending=True, stable=True)
        prob = torch.softmax(v, 0)
        if T == 0:
            token.append(order[:1]), conf.append(prob[order[:1]]), kept.append(1)
            continue
        inside = int((v > -math.inf).sum())
        if k > 0:
            inside = min(inside, int(k))
        q = torch.softmax(v[order[:inside]] / T, 0)    # of what is kept so far
        if p < 1:
            at = q.cumsum(0)
            inside = min(inside, int(torch.searchsorted(at, p * at[-1:])) + 1)
        if m > 0:
            inside = max(1, min(inside, int((q[:inside] >= m * q[0]).sum())))
        at = q[:inside].cumsum(0)
        j = min(int(torch.searchsorted(at, s["u"][r].double() * at[-1:], right=True)), inside - 1)
        token.append(order[j: j + 1]), conf.append(prob[order[j: j + 1]]), kept.append(inside)
    return dict(token=torch.cat(token).to(torch.int32), conf=torch.cat(conf), kept=torch.tensor(kept, dtype=torch.int32, device="cuda"))


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "extend":
        P, N = c["page"], c["page"] * c["width"]
        table, lens, new, free = (s[k].tolist() for k in ("table", "lens", "new", "free"))
        n_free, idx = s["n_free"].item(), s["idx"].tolist()
        top, want, rows, at, offsets = n_free, 0, 0, 0, [0]
        for b in range(c["B"]):
            need = _ceil(lens[b] + new[b], P) - _ceil(lens[b], P)
            if lens[b] + new[b] <= N:
                want, rows = want + need, rows + new[b]
                if (need == 0 or want <= n_free) and rows <= s["rows"]:
                    for j in range(_ceil(lens[b], P), _ceil(lens[b] + new[b], P)):
                        top -= 1
                        table[b][j] = free[top]
                    for i in range(new[b]):
                        idx[at + i] = b * N + lens[b] + i
                    at, lens[b] = at + new[b], lens[b] + new[b]
            offsets.append(at)
        out = dict(table=table, lens=lens, n_free=[top], offsets=offsets, idx=idx, n=[at])
        return {k: torch.tensor(v, dtype=torch.int32, device="cuda") for k, v in out.items()}
    if c["op"] == "truncate":
        table, lens, keep, free = (s[k].tolist() for k in ("table", "lens", "keep", "free"))
        top = s["n_free"].item()
        for b in range(c["B"]):
            n = min(keep[b], lens[b])
            for j in range(_ceil(n, c["page"]), _ceil(lens[b], c["page"])):
                free[top] = table[b][j]
                top += 1
            lens[b] = n
        return {k: torch.tensor(v, dtype=torch.int32, device="cuda") for k, v in dict(free=free, lens=lens, n_free=[top]).items()}
    if c["op"] == "rope":
        turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["pos"].double()[:, None] * s["freq"][None])[:, None]
        out = {}
        for name in ("q", "k"):
            y = s[name].double()
            n = c["rot"]
            pair = y[..., :n].unflatten(-1, (-1, 2)) if c["interleaved"] else y[..., :n].unflatten(-1, (2, -1)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            y[..., :n] = (z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            out[name] = y
        return out
    if c["op"] == "adapters":
        y = s["y"].double()
        offs, which, ranks = (s[k].tolist() for k in ("offsets", "which", "ranks"))
        for b in range(c["B"]):
            i = which[b]
            if i >= 0:
                rows, r = slice(offs[b], offs[b + 1]), ranks[i]
                t = torch.einsum("mk,rk->mr", s["x"][rows].double(), s["a"][i, :r].double())
                y[rows] += torch.einsum("mr,nr->mn", t, s["b"][i, :, :r].double()) * s["scale"][i].double()
        return y
    return _exact_sample(s)
