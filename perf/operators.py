"""The operators of a serving step over a paged cache, as measured cases.

Three operators, as a serving program of a Qwen3-shaped decoder calls them between its projections:

* ``append``    -- per-head RMSNorm of q and k, rotary embedding, and the append of k and v to a paged
                   cache, for a ragged batch of new tokens;
* ``attention`` -- causal grouped-query attention of those tokens over the paged cache;
* ``sample``    -- temperature, top-k, top-p and min-p sampling from given random numbers.

Head counts, head size, rotary base and vocabulary are those of the Qwen3 decoders the repository
runs (32 q heads, 8 kv heads of 128, vocabulary 151936) and a few other groupings.
"""
import math

import torch

own = False

D = 128
THETA = 1e6
EPS = 1e-6
SCALE = 1.0 / math.sqrt(D)
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
FIXED = 2.0 ** 40       # the unit weight of sampling
U24 = 1 << 24           # steps of top_p and of the random numbers


def _dev():
    return torch.device("cuda") if torch.cuda.is_available() else torch.device("cpu")


# ---------------------------------------------------------------------------------------------
# the cases

# append and attention: requests with chunks of "long" new tokens and "long_len" cached ones (with
# the new), and "short" requests of one new token each

def listed():
    return [
        # one request that decodes: the append between q|k|v and attention, where latency counts
        dict(name="append_1", op="append", type="f16", Hq=32, Hkv=8, page=16, long="", short=1,
             short_len=2048, ragged=0),
        # a mixed serving step: rows that decode beside prompt chunks of odd lengths
        dict(name="append_mixed", op="append", type="bf16", Hq=32, Hkv=8, page=64,
             long="509,771,130", long_len="4096,771,9001", short=61, short_len=2000, ragged=1),
        # a long prompt at once
        dict(name="append_8192", op="append", type="f16", Hq=32, Hkv=8, page=128, long="8192",
             long_len="8192", short=0, short_len=0, ragged=0),
        # one request that decodes at a context of 2048
        dict(name="attention_1x2048", op="attention", type="f16", Hq=32, Hkv=8, page=16, long="",
             short=1, short_len=2048, ragged=0),
        # 32 requests that decode at contexts up to 8192
        dict(name="attention_32x8192", op="attention", type="f16", Hq=32, Hkv=8, page=16, long="",
             short=32, short_len=8192, ragged=1),
        # one request that decodes at a very long, odd context
        dict(name="attention_1x65537", op="attention", type="bf16", Hq=32, Hkv=8, page=64, long="",
             short=1, short_len=65537, ragged=0),
        # a mixed serving step: 31 rows that decode and one prompt chunk
        dict(name="attention_mixed", op="attention", type="f16", Hq=32, Hkv=8, page=32, long="509",
             long_len="4093", short=31, short_len=4096, ragged=1),
        # a prompt chunk deep in a long context
        dict(name="attention_1024_of_16384", op="attention", type="bf16", Hq=32, Hkv=8, page=128,
             long="1024", long_len="16384", short=0, short_len=0, ragged=0),
        # a long prompt at once
        dict(name="attention_8192", op="attention", type="f16", Hq=32, Hkv=8, page=64, long="8192",
             long_len="8192", short=0, short_len=0, ragged=0),
        # the next token of one request
        dict(name="sample_1", op="sample", type="f16", M=1, V=151936, open=0.0),
        # the next tokens of a full batch, with settings of their own
        dict(name="sample_64", op="sample", type="f16", M=64, V=151936, open=0.0),
        # many rows of a smaller, odd vocabulary in 32 bits, some of them not cut at all
        dict(name="sample_257x32003", op="sample", type="f32", M=257, V=32003, open=0.1),
    ]


def _loguniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def _text(numbers):
    return ",".join(map(str, numbers))


def _numbers(text):
    return [int(x) for x in text.split(",") if x]


_LIMIT = {}


def draw(rng):
    if not _LIMIT:
        for c in listed():
            w = work(c)
            for k in w:
                _LIMIT[c["op"], k] = max(w[k], _LIMIT.get((c["op"], k), 0))
    op = rng.choice(["append", "attention", "attention", "sample"])
    while True:
        if op == "sample":
            c = dict(op=op, type=rng.choice(["f16", "bf16", "f32"]), M=_loguniform(rng, 1, 300),
                     V=_loguniform(rng, 1000, 200000), open=rng.choice([0.0, 0.0, 0.2]))
        else:
            Hkv = rng.choice([1, 2, 4, 8, 8])
            G = rng.choice([1, 2, 4, 4, 5, 7, 8])
            longs = [_loguniform(rng, 2, 4096) for _ in range(rng.choice([0, 0, 1, 1, 2, 5]))]
            c = dict(op=op, type=rng.choice(["f16", "bf16"]), Hq=G * Hkv, Hkv=Hkv,
                     page=rng.choice([16, 32, 64, 128, 256]), long=_text(longs),
                     long_len=_text(n + rng.choice([0, _loguniform(rng, 1, 20000)])
                                    for n in longs),
                     short=_loguniform(rng, 1, 100) if not longs else rng.choice([0, 1, 9, 40]),
                     short_len=_loguniform(rng, 1, 40000), ragged=rng.choice([0, 1, 1]))
        w = work(c)
        if all(w[k] <= _LIMIT[op, k] for k in w) and (
                op != "append" or sum(_lengths(c)[1]) * c["Hkv"] <= 8 * 80000):
            return c


def _lengths(c, seed=None):
    """(new tokens, cached tokens with the new ones) of every request of a case.  Ragged short rows
    have from 1/16 of short_len to all of it, evenly spread (shuffled by the seed)."""
    n, L = _numbers(c["long"]), _numbers(c.get("long_len", ""))
    S = c["short"]
    lens = [c["short_len"]] * S
    if c["ragged"] and S > 1:
        lens = [max(1, int(c["short_len"] * (1 + 15 * (i + 1) / S) / 16)) for i in range(S)]
    order = list(range(len(n) + S))
    if seed is not None:
        g = torch.Generator().manual_seed(seed)
        order = torch.randperm(len(order), generator=g).tolist()
    n, L = n + [1] * S, L + lens
    return [n[i] for i in order], [L[i] for i in order]


def work(c):
    if c["op"] == "sample":
        size = 4 if c["type"] == "f32" else 2
        # the logits once, the settings of each row, its token and probability; an exponential,
        # a scaling, a sum and the comparison of the cut for every logit
        return {"bytes": c["M"] * (c["V"] * size + 28), "flops": 4 * c["M"] * c["V"]}
    n, L = _lengths(c)
    T, B, Hq, Hkv = sum(n), len(n), c["Hq"], c["Hkv"]
    tables = 4 * (2 * B + 1) + 4 * sum(-(-x // c["page"]) for x in L)
    if c["op"] == "append":
        # every head vector read and written once; norm (4) and rotation (3) of q and k
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * D * 2 + tables, "flops": 7 * T * (Hq + Hkv) * D}
    pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(n, L))
    return {"bytes": 2 * T * Hq * D * 2 + 2 * sum(L) * Hkv * D * 2 + tables,
            "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------------------------------------
# the inputs

def _inputs(c, seed):
    """What the operators read, from the seed alone."""
    dev = _dev()
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = TYPES[c["type"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=dev)

    if c["op"] == "sample":
        M, V = c["M"], c["V"]
        # a language model's logits: a wide body, and a head of a few dozen tokens above it
        x = 1.5 * normal(M, V)
        head = min(40, V)
        at = torch.rand((M, V), generator=g, device=dev).topk(head, dim=1).indices
        top = 14.0 - 0.35 * torch.arange(head, device=dev) + 0.5 * normal(M, head)
        x.scatter_(1, at, top)
        # settings as requests bring them: most rows cut by some of the three, greedy ones, and
        # (with the share "open") rows that are not cut
        r = torch.rand((6, M), generator=g, device=dev)
        T = 0.6 + 0.5 * r[0]
        T = torch.where(r[5] > 0.95, torch.zeros_like(T), T)
        k = torch.where(r[1] < 0.5, (5 + 60 * r[1] * 2).to(torch.int32),
                        torch.zeros((M,), dtype=torch.int32, device=dev)).to(torch.int32)
        p = torch.where((r[2] < 0.6) | (k == 0), 0.7 + 0.25 * r[2], torch.ones_like(T))
        m = torch.where(r[3] < 0.3, 0.02 + 0.2 * r[3], torch.zeros_like(T))
        free = r[4] < c["open"]
        k, p, m = k * (~free), torch.where(free, torch.ones_like(p), p), m * (~free)
        return dict(logits=x.to(dt), T=T.contiguous(), k=k.to(torch.int32).contiguous(),
                    p=p.contiguous(), m=m.contiguous(),
                    u=torch.rand((M,), generator=g, device=dev))

    n, L = _lengths(c, seed)
    Hq, Hkv, P, T, B = c["Hq"], c["Hkv"], c["page"], sum(n), len(n)
    used = [-(-x // P) for x in L]
    pages = sum(used) + 3
    ids = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((B, max(used)), -1, dtype=torch.int32)
    at = 0
    for b, x in enumerate(used):
        table[b, :x] = ids[at:at + x]
        at += x
    start = torch.zeros((B + 1,), dtype=torch.int32)
    start[1:] = torch.cumsum(torch.tensor(n), 0)
    s = dict(table=table.to(dev), start=start.to(dev),
             kv_len=torch.tensor(L, dtype=torch.int32).to(dev), n=n, L=L)
    if c["op"] == "append":
        s["qkv"] = (2.0 * normal(T, (Hq + 2 * Hkv) * D)).to(dt)
        s["qw"] = (1.0 + 0.1 * normal(D)).to(dt)
        s["kw"] = (1.0 + 0.1 * normal(D)).to(dt)
    else:
        s["q"] = (1.5 * normal(T, Hq, D)).to(dt)
    s["kc"] = normal(pages, Hkv, P, D).to(dt)
    s["vc"] = normal(pages, Hkv, P, D).to(dt)
    if c["op"] == "attention":
        # the first token of a request draws attention, as it does in trained models
        first = s["table"][:, 0].long()
        s["kc"][first, :, 0] *= 2
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["op"] == "sample":
        M = case["M"]
        s["out"] = torch.empty((M,), dtype=torch.int32, device=_dev())
        s["prob"] = torch.empty((M,), dtype=torch.float32, device=_dev())
    elif case["op"] == "append":
        s["q_out"] = torch.empty((sum(s["n"]), case["Hq"], D), dtype=s["qkv"].dtype, device=_dev())
    else:
        s["out"] = torch.empty_like(s["q"])
    if own and case["op"] != "sample":
        # the cache's description and the workspace, which a serving program keeps for its buffers
        from paper_2605_08755_gb300 import _lib
        s["cache"] = _lib.PagedCache(s["kc"], s["vc"], s["table"], s["start"], s["kv_len"])
        if case["op"] == "attention":
            s["max_q"] = max(s["n"])
            s["ws"] = _lib.paged_attention_workspace(sum(s["n"]), len(s["n"]), s["max_q"],
                                                     case["Hq"], case["Hkv"], _dev())
    return s


# ---------------------------------------------------------------------------------------------
# one pass

def run(s):
    c = s["case"]
    if own:
        from paper_2605_08755_gb300 import _lib
        if c["op"] == "append":
            q = _lib.laq_paged_append(s["qkv"], s["cache"], c["Hq"], THETA, EPS, q_norm_w=s["qw"],
                                      k_norm_w=s["kw"], q_out=s["q_out"])
            return {"q": q, "k_cache": s["kc"], "v_cache": s["vc"]}
        if c["op"] == "attention":
            return _lib.laq_paged_attention(s["q"], s["cache"], s["max_q"], SCALE, s["ws"],
                                            out=s["out"])
        token = _lib.laq_sample(s["logits"], s["u"], temperature=s["T"], top_k=s["k"],
                                top_p=s["p"], min_p=s["m"], out=s["out"], p_out=s["prob"])
        return {"token": token, "prob": s["prob"]}
    if c["op"] == "append":
        return _plain_append(s, c)
    if c["op"] == "attention":
        return _plain_attention(s, c)
    return _plain_sample(s)


def _plain_append(s, c):
    Hq, Hkv, P, dt, dev = c["Hq"], c["Hkv"], c["page"], s["qkv"].dtype, s["qkv"].device
    T = s["qkv"].shape[0]
    t = torch.arange(T, device=dev)
    b = torch.searchsorted(s["start"][1:].long(), t, right=True)
    end = s["start"].long()[1:][b]
    pos = s["kv_len"].long()[b] - (end - t)
    x = s["qkv"].float().view(T, Hq + 2 * Hkv, D)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], s["qkv"].view(T, Hq + 2 * Hkv, D)[:, Hq + Hkv:]
    # the angle as a fraction of a turn, in 40 bits of whole-number arithmetic: pos * f mod 1
    turn = torch.tensor([round(THETA ** (-2.0 * i / D) / (2 * math.pi) * 2 ** 40)
                         for i in range(D // 2)], device=dev)
    phase = ((pos[:, None] * turn[None]) & (2 ** 40 - 1)).float() * 2.0 ** -40
    cos, sin = torch.cos(2 * math.pi * phase)[:, None], torch.sin(2 * math.pi * phase)[:, None]

    def turned(h, w):
        h = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * w.float()
        lo, hi = h[..., :D // 2], h[..., D // 2:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(dt)

    page = s["table"].long()[b, pos // P]
    s["kc"][page, :, pos % P] = turned(k, s["kw"])
    s["vc"][page, :, pos % P] = v
    return {"q": turned(q, s["qw"]), "k_cache": s["kc"], "v_cache": s["vc"]}


def _plain_attention(s, c):
    Hq, Hkv, P, dev = c["Hq"], c["Hkv"], c["page"], s["q"].device
    G, at, outs = Hq // Hkv, 0, []
    for b, (n, L) in enumerate(zip(s["n"], s["L"])):
        page = s["table"][b, :-(-L // P)].long()
        k = s["kc"][page].transpose(0, 1).reshape(Hkv, -1, D)[:, :L].float()
        v = s["vc"][page].transpose(0, 1).reshape(Hkv, -1, D)[:, :L].float()
        q = s["q"][at:at + n].float().view(n, Hkv, G, D).permute(1, 2, 0, 3).reshape(Hkv, G * n, D)
        x = torch.matmul(q, k.transpose(1, 2)) * SCALE
        if n > 1:
            pos = torch.arange(L - n, L, device=dev).repeat(G)
            x.masked_fill_(torch.arange(L, device=dev)[None] > pos[:, None], float("-inf"))
        x = torch.exp(x - x.amax(-1, keepdim=True))
        o = torch.matmul(x, v) / x.sum(-1, keepdim=True)
        outs.append(o.view(Hkv, G, n, D).permute(2, 0, 1, 3).reshape(n, Hq, D).to(s["q"].dtype))
        at += n
    return torch.cat(outs)


def _plain_sample(s):
    x = s["logits"].float()
    M, V = x.shape
    x = torch.where(torch.isnan(x), torch.full_like(x, float("-inf")), x)
    top = x.amax(1, keepdim=True)
    T = s["T"][:, None]
    greedy = ~(T > 0)
    # weights as whole numbers (2^40 for the largest), so that no sum depends on its order
    e = torch.exp((x - top) / torch.where(greedy, torch.ones_like(T), T))
    e = torch.where(x == top, torch.ones_like(e), torch.where(greedy, torch.zeros_like(e), e))
    w = (e * FIXED).to(torch.int64)
    by = torch.sort(x, dim=1, descending=True, stable=True).indices
    ws = w.gather(1, by)
    rank = torch.arange(V, device=x.device)[None]
    k = s["k"].long()[:, None]
    keep = (k <= 0) | (rank < k)
    ws = ws * keep
    cum = torch.cumsum(ws, 1)

    def part(mass, f):   # floor(mass * f), f in steps of 2^-24
        f = (f * U24).to(torch.int64)
        return (mass >> 24) * f + (((mass & (U24 - 1)) * f) >> 24)

    p = s["p"][:, None]
    keep &= (p >= 1) | (rank == 0) | (cum - ws < part(cum[:, -1:], p.clamp(0, 1)))
    m = s["m"][:, None].clamp(0, 1)
    keep &= (ws >= (m * FIXED).to(torch.int64)) | (rank == 0)
    keep &= ~greedy | (rank == 0)
    kept = torch.zeros_like(keep).scatter_(1, by, keep)
    w = w * kept
    cum = torch.cumsum(w, 1)
    total = cum[:, -1:]
    token = (cum <= part(total, s["u"][:, None])).sum(1, keepdim=True)
    prob = w.gather(1, token).float() / total.float()
    return {"token": token[:, 0].to(torch.int32), "prob": prob[:, 0]}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "sample":
        return _exact_sample(s)
    start, table = s["start"].tolist(), s["table"].tolist()
    P, Hq, Hkv = case["page"], case["Hq"], case["Hkv"]
    G = Hq // Hkv
    dev = s["kc"].device
    if case["op"] == "append":
        x = s["qkv"].double().view(-1, Hq + 2 * Hkv, D)
        pos, page, slot = [], [], []
        for b, (n, L) in enumerate(zip(s["n"], s["L"])):
            for p in range(L - n, L):
                pos.append(p)
                page.append(table[b][p // P])
                slot.append(p % P)
        freq = torch.tensor([THETA ** (-2 * i / D) for i in range(D // 2)], dtype=torch.float64,
                            device=dev)
        a = torch.tensor(pos, dtype=torch.float64, device=dev)[:, None] * freq
        z = torch.polar(torch.ones_like(a), a)[:, None]

        def turned(h, w):
            h = h / torch.sqrt(torch.mean(h ** 2, -1, keepdim=True) + EPS) * w.double()
            h = torch.complex(h[..., :D // 2].contiguous(), h[..., D // 2:].contiguous()) * z
            return torch.cat([h.real, h.imag], -1)

        kc, vc = s["kc"].double(), s["vc"].double()
        page, slot = torch.tensor(page, device=dev), torch.tensor(slot, device=dev)
        kc[page, :, slot] = turned(x[:, Hq:Hq + Hkv], s["kw"])
        vc[page, :, slot] = x[:, Hq + Hkv:]
        return {"q": turned(x[:, :Hq], s["qw"]), "k_cache": kc, "v_cache": vc}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=dev)
    for b, (n, L) in enumerate(zip(s["n"], s["L"])):
        tok = torch.arange(L, device=dev)
        page = s["table"][b].long()[tok // P]
        for h in range(Hkv):
            k, v = s["kc"][page, h, tok % P].double(), s["vc"][page, h, tok % P].double()
            for i0 in range(0, n, 1024):
                i1 = min(n, i0 + 1024)
                end = L - n + i1
                q = s["q"][start[b] + i0:start[b] + i1, h * G:(h + 1) * G].double()
                x = torch.einsum("igd,td->igt", q * SCALE, k[:end])
                seen = torch.arange(L - n + i0, end, device=dev)[:, None] >= tok[None, :end]
                x = torch.where(seen[:, None], x, -math.inf)
                x = torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
                out[start[b] + i0:start[b] + i1, h * G:(h + 1) * G] = \
                    torch.einsum("igt,td->igd", x, v[:end])
    return out


def _exact_sample(s):
    """The tokens by the definition in 64 bits, row by row; None where a cut or the drawn number falls
    so close to a boundary that 32-bit weights may decide it the other way."""
    near = 2e-7
    tokens, probs = [], []
    for m in range(s["logits"].shape[0]):
        x = s["logits"][m].double()
        T, k, p, lo, u = (s[j][m].item() for j in ("T", "k", "p", "m", "u"))
        if not T > 0:
            tokens.append(int((x == x.max()).nonzero()[0, 0]))
            probs.append(1.0)
            continue
        w = torch.softmax(x / T, 0)
        w, by = torch.sort(w, descending=True, stable=True)
        if k > 0:
            w, by = w[:k], by[:k]
        if p < 1:
            part = torch.cumsum(w, 0) / w.sum()
            if (part - p).abs().min() < near:
                return {"token": None, "prob": None}
            last = int((part < p).sum())
            w, by = w[:last + 1], by[:last + 1]
        if lo > 0:
            if (w / w[0] / lo - 1).abs().min() < 2e-6:
                return {"token": None, "prob": None}
            keep = w >= lo * w[0]
            w, by = w[keep], by[keep]
        by, order = torch.sort(by)
        w = w[order] / w.sum()
        cum = torch.cumsum(w, 0)
        if cum.numel() > 1 and (cum[:-1] - u).abs().min() < near:
            return {"token": None, "prob": None}
        j = min(int((cum <= u).sum()), cum.numel() - 1)
        tokens.append(int(by[j]))
        probs.append(float(w[j]))
    dev = s["logits"].device
    return {"token": torch.tensor(tokens, dtype=torch.int32, device=dev),
            "prob": torch.tensor(probs, dtype=torch.float64, device=dev)}
