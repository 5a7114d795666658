"""Cases of one decode step of a dispatched batch, in plain torch and through
``driftsched``.

A case is one of three operators:

  attention  ``decode_attention``: 1 to 16 new tokens per request over a paged
             key-value cache, whole or through a window with sink tokens, with
             or without the attention weight summed per cached token
  evict      ``cache_evict``: requests that outgrew their token budget keep the
             tokens of the largest accumulated weight, in fresh pages
  verify     ``verify_draft``: drafted tokens against the target's
             probabilities, from given random numbers

With ``own`` false ``run`` computes the operator in elementary operations in
32 bits (64 in the long sums of the verification); with ``own`` true it makes
the calls of a serving program.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
ACCEPT = 0.8          # share of drafted tokens that a target accepts, one by one


def listed():
    return [
        # one short chat request, one new token: bound by launches and latency
        {"name": "attention_single", "op": "attention", "rows": 1, "lo": 150, "hi": 200, "page": 16, "n_kv": 2,
         "group": 4, "dim": 64, "tokens": 1, "q": "bf16", "kv": "bf16", "window": 0, "sinks": 0, "mass": False},
        # a dispatch batch of 32 chat requests, every query head with keys of its own
        {"name": "attention_batch", "op": "attention", "rows": 32, "lo": 64, "hi": 2048, "page": 16, "n_kv": 16,
         "group": 1, "dim": 128, "tokens": 1, "q": "bf16", "kv": "bf16", "window": 0, "sinks": 0, "mass": False},
        # four drafted tokens per request to be verified, sliding window with sinks
        {"name": "attention_drafts", "op": "attention", "rows": 16, "lo": 500, "hi": 6000, "page": 32, "n_kv": 4,
         "group": 8, "dim": 128, "tokens": 5, "q": "f16", "kv": "f16", "window": 1024, "sinks": 4, "mass": False},
        # a loaded server: 8-bit cache, weights summed for a later eviction
        {"name": "attention_mass8", "op": "attention", "rows": 48, "lo": 2000, "hi": 8192, "page": 64, "n_kv": 8,
         "group": 4, "dim": 128, "tokens": 1, "q": "bf16", "kv": "e4m3", "window": 0, "sinks": 0, "mass": True},
        # three long-context requests: few rows, split over the cache's length
        {"name": "attention_long", "op": "attention", "rows": 3, "lo": 40000, "hi": 131072, "page": 64, "n_kv": 8,
         "group": 4, "dim": 128, "tokens": 1, "q": "bf16", "kv": "bf16", "window": 0, "sinks": 0, "mass": False},
        # two short answers that ran over their budgets
        {"name": "evict_small", "op": "evict", "rows": 2, "lo": 300, "hi": 700, "page": 16, "n_kv": 2, "dim": 64,
         "kv": "bf16", "sinks": 4, "recent": 32, "keep_lo": 0.4, "keep_hi": 0.9},
        # a dispatch batch after drift: some requests within their budgets, most above
        {"name": "evict_batch", "op": "evict", "rows": 32, "lo": 2048, "hi": 6144, "page": 16, "n_kv": 8, "dim": 128,
         "kv": "f16", "sinks": 4, "recent": 256, "keep_lo": 0.5, "keep_hi": 1.05},
        # long contexts cut to about half
        {"name": "evict_long", "op": "evict", "rows": 3, "lo": 60000, "hi": 100000, "page": 64, "n_kv": 8, "dim": 128,
         "kv": "bf16", "sinks": 16, "recent": 1024, "keep_lo": 0.4, "keep_hi": 0.6},
        # one request, three drafted tokens
        {"name": "verify_single", "op": "verify", "rows": 1, "drafts": 3, "vocab": 32000, "type": "f32", "dist": True},
        # a dispatch batch, a large vocabulary
        {"name": "verify_batch", "op": "verify", "rows": 32, "drafts": 4, "vocab": 128000, "type": "f32", "dist": True},
        # drafts copied from the prompt: no draft distribution, odd vocabulary, 16-bit probabilities
        {"name": "verify_copied", "op": "verify", "rows": 200, "drafts": 7, "vocab": 50257, "type": "bf16", "dist": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "evict", "verify"])
    if op == "attention":
        kv = rng.choice(["bf16", "f16", "e4m3"])
        q = rng.choice(["bf16", "f16"]) if kv == "e4m3" else kv
        n_kv, group, dim = rng.choice([1, 2, 3, 4, 8, 16]), rng.choice([1, 2, 3, 4, 5, 8, 16]), rng.choice([64, 80, 96, 128, 256])
        tokens = rng.choice([1, 1, 2, 3, 5, 8])
        rows = _log(rng, 1, 64)
        most = min(131072, max(16, int(2.0e8 / (rows * n_kv * dim))))   # tokens per row: below the largest listed cache
        hi = _log(rng, 1, most)
        lo = max(1, int(hi * rng.uniform(0.02, 1.0)))
        window = _log(rng, 16, 4096) if rng.random() < 0.3 else 0
        return {"op": op, "rows": rows, "lo": lo, "hi": hi, "page": rng.choice([8, 16, 24, 32, 64, 128]), "n_kv": n_kv,
                "group": group, "dim": dim, "tokens": tokens, "q": q, "kv": kv, "window": window,
                "sinks": rng.choice([0, 1, 4, 33]) if window else 0, "mass": rng.random() < 0.4}
    if op == "evict":
        n_kv, dim = rng.choice([1, 2, 4, 8]), rng.choice([64, 80, 128, 256])
        rows = _log(rng, 1, 64)
        most = min(100000, max(64, int(2.0e8 / (rows * n_kv * dim))))
        hi = _log(rng, 8, most)
        lo = max(1, int(hi * rng.uniform(0.1, 1.0)))
        keep = rng.uniform(0.1, 0.9)
        return {"op": op, "rows": rows, "lo": lo, "hi": hi, "page": rng.choice([8, 16, 24, 64]), "n_kv": n_kv, "dim": dim,
                "kv": rng.choice(["bf16", "f16", "e4m3"]), "sinks": rng.choice([0, 1, 4, 16]),
                "recent": min(_log(rng, 1, 1024), hi), "keep_lo": keep, "keep_hi": min(1.1, keep + rng.uniform(0.05, 0.5))}
    rows, vocab = _log(rng, 1, 200), _log(rng, 100, 160000)
    drafts = rng.choice([0, 1, 2, 3, 4, 5, 7])
    if rows * (drafts + 1) * vocab > 9e7:
        rows = max(1, int(9e7 / ((drafts + 1) * vocab)))
    return {"op": op, "rows": rows, "drafts": drafts, "vocab": vocab, "type": rng.choice(["f32", "f16", "bf16"]),
            "dist": rng.random() < 0.6}


# ---- inputs -----------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _pool(pages, page, n_kv, dim, kind, g):
    shape = (pages, page, n_kv, dim)
    x = torch.empty(shape, dtype=TYPES["bf16" if kind == "e4m3" else kind], device="cuda").normal_(generator=g)
    return (x * 8).to(TYPES[kind]) if kind == "e4m3" else x


def _lengths(rows, lo, hi, g):
    n = torch.randint(lo, hi + 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
    n[0] = hi
    return n


def _cache(case, g):
    """A pool in which the requests' pages lie scattered; twice as many requests
    as rows, the batch being some of them in dispatch order."""
    rows, page, hi = case["rows"], case["page"], case["hi"]
    per = -(-hi // page)
    n_req = rows + 2
    lens = _lengths(rows, case["lo"], hi, g)
    full = torch.zeros(n_req, dtype=torch.int32, device="cuda")
    order = torch.randperm(n_req, generator=g, device="cuda")[:rows].to(torch.int32)
    full[order.long()] = lens
    table = torch.zeros((n_req, per), dtype=torch.int32, device="cuda")
    table[order.long()] = torch.randperm(rows * per, generator=g, device="cuda").to(torch.int32).view(rows, per)
    s = {"case": case, "rows": order, "lens": full, "table": table, "max_len": hi,
         "k": _pool(rows * per, page, case["n_kv"], case["dim"], case["kv"], g),
         "v": _pool(rows * per, page, case["n_kv"], case["dim"], case["kv"], g)}
    if case["kv"] == "e4m3":
        s["k_scale"] = torch.rand(case["n_kv"], generator=g, device="cuda") * 0.1 + 0.1
        s["v_scale"] = torch.rand(case["n_kv"], generator=g, device="cuda") * 0.1 + 0.1
    if own:
        from paper_2606_02982_amd import driftsched as ds
        s["cache"] = ds.kv_cache(s["k"], s["v"], table, full, s.get("k_scale"), s.get("v_scale"))
    return s


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "attention":
        s = _cache(case, g)
        heads = case["n_kv"] * case["group"]
        s["q"] = (2 * torch.randn((case["rows"], case["tokens"], heads, case["dim"]), generator=g, device="cuda")).to(TYPES[case["q"]])
        if case["mass"]:
            s["mass"] = torch.rand((case["rows"] + 2, case["n_kv"], case["hi"]), generator=g, device="cuda")
        return s
    if case["op"] == "evict":
        s = _cache(case, g)
        rows, page, hi = case["rows"], case["page"], case["hi"]
        # weights as attention leaves them: a few tokens hold most, many are equal (never looked at)
        m = torch.rand((rows + 2, case["n_kv"], hi), generator=g, device="cuda")
        s["mass"] = torch.where(m < 0.2, torch.zeros_like(m), (3 * torch.randn(m.shape, generator=g, device="cuda")).exp())
        share = case["keep_lo"] + (case["keep_hi"] - case["keep_lo"]) * torch.rand(rows + 2, generator=g, device="cuda", dtype=torch.float64)
        s["budget"] = s["lens"].double() * share + 0.37
        most = min(hi, max(int(hi * case["keep_hi"]) + 1, case["sinks"] + case["recent"]))
        per = -(-most // page)
        s["dst_k"] = torch.zeros((rows * per, page, case["n_kv"], case["dim"]), dtype=s["k"].dtype, device="cuda")
        s["dst_v"] = torch.zeros_like(s["dst_k"])
        s["dst_table"] = torch.randperm(rows * per, generator=g, device="cuda").to(torch.int32).view(rows, per)
        s["dst_lens"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
        s["mass_out"] = torch.zeros_like(s["mass"])
        s["kept"] = torch.full((rows, case["n_kv"], per * page), -1, dtype=torch.int32, device="cuda")
        if own:
            from paper_2606_02982_amd import driftsched as ds
            s["dst"] = ds.kv_cache(s["dst_k"], s["dst_v"], s["dst_table"], s["dst_lens"], s.get("k_scale"), s.get("v_scale"))
        return s
    rows, n, vocab, kind = case["rows"], case["drafts"], case["vocab"], TYPES[case["type"]]

    def peaked(shape):
        # one token stands out in each position, as in text
        x = 2 * torch.randn(shape, generator=g, device="cuda")
        top = torch.randint(0, shape[-1], shape[:-1] + (1,), generator=g, device="cuda")
        return torch.softmax(x.scatter(-1, top, math.log(shape[-1]) + 3.5), -1)

    p = peaked((rows, n + 1, vocab))
    s = {"case": case, "target": p.to(kind), "draft": None}
    if case["dist"]:
        q = ACCEPT * p[:, :n] + (1 - ACCEPT) * peaked((rows, n, vocab)) if n else p[:, :0]
        s["draft"] = q.to(kind).contiguous()
    else:
        q = p[:, :n]
    picks = torch.multinomial(q.reshape(-1, vocab), 1, generator=g) if n else torch.zeros(0, device="cuda")
    s["tokens"] = picks.view(rows, n).to(torch.int32)
    s["u"] = torch.rand((rows, n), generator=g, device="cuda")
    s["u_sample"] = torch.rand(rows, generator=g, device="cuda")
    s["n_draft"] = torch.randint(max(0, n - 2), n + 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
    s["rows"] = torch.randperm(rows + 3, generator=g, device="cuda")[:rows].to(torch.int32)
    s["observed"] = torch.randint(0, 500, (rows + 3,), generator=g, device="cuda", dtype=torch.int32)
    s["lens"] = torch.randint(0, 2000, (rows + 3,), generator=g, device="cuda", dtype=torch.int32)
    return s


# ---- one pass ---------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"attention": _own_attention, "evict": _own_evict, "verify": _own_verify}[op](state)
    return {"attention": _attention, "evict": _evict, "verify": _verify}[op](state)


def _values(x):
    return x.float() if x.dtype == torch.float8_e4m3fn else x


def _own_attention(s):
    from paper_2606_02982_amd import driftsched as ds
    c = s["case"]
    out = ds.decode_attention(s["q"], s["cache"], rows=s["rows"], window=c["window"], sinks=c["sinks"],
                              max_len=s["max_len"], mass=s.get("mass"))
    return {"out": out, "mass": s["mass"]} if c["mass"] else {"out": out}


def _own_evict(s):
    from paper_2606_02982_amd import driftsched as ds
    c = s["case"]
    ds.cache_evict(s["cache"], s["dst"], s["budget"], s["mass"], rows=s["rows"], sinks=c["sinks"], recent=c["recent"],
                   max_len=s["max_len"], mass_out=s["mass_out"], kept=s["kept"])
    return {"k": _values(s["dst_k"]), "v": _values(s["dst_v"]), "len": s["dst_lens"], "kept": s["kept"], "mass": s["mass_out"]}


def _own_verify(s):
    from paper_2606_02982_amd import driftsched as ds
    out, emitted = ds.verify_draft(s["target"], s["draft"], s["tokens"], s["u"], s["u_sample"], n_draft=s["n_draft"],
                                   rows=s["rows"], observed=s["observed"], lens=s["lens"])
    return {"tokens": out, "emitted": emitted, "observed": s["observed"], "lens": s["lens"]}


def _attention(s):
    c, rows = s["case"], s["rows"].long()
    n_kv, group, t, page = c["n_kv"], c["group"], c["tokens"], c["page"]
    n, dev = s["lens"][rows], s["q"].device
    j = torch.arange(s["max_len"], device=dev)
    where = s["table"][rows].long()[:, j // page], (j % page)[None, :]
    k = s["k"][where].float()                                            # rows, length, n_kv, dim
    if "k_scale" in s:
        k = k * s["k_scale"][:, None]
    q = s["q"].float().view(c["rows"], t, n_kv, group, c["dim"]).permute(0, 2, 1, 3, 4).reshape(c["rows"], n_kv, t * group, c["dim"])
    x = torch.matmul(q.contiguous(), k.permute(0, 2, 3, 1).contiguous()) * (1 / math.sqrt(c["dim"]))
    del k
    at = (n[:, None] - t + torch.arange(t, device=dev))[:, :, None]      # rows, tokens, 1: the queries' positions
    seen = j <= at
    if c["window"]:
        seen = seen & ((j > at - c["window"]) | (j < c["sinks"]))
    seen = seen[:, None, :, None, :].expand(-1, n_kv, -1, group, -1).reshape(c["rows"], n_kv, t * group, -1)
    x = torch.where(seen, x, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = x.sum(-1, keepdim=True)
    x = x / torch.where(total == 0, 1.0, total)
    v = torch.where((j < n[:, None])[:, :, None, None], s["v"][where].float(), 0.0)
    if "v_scale" in s:
        v = v * s["v_scale"][:, None]
    out = torch.matmul(x, v.permute(0, 2, 1, 3).contiguous())
    out = out.view(c["rows"], n_kv, t, group, c["dim"]).permute(0, 2, 1, 3, 4).reshape(c["rows"], t, n_kv * group, c["dim"]).to(s["q"].dtype)
    if not c["mass"]:
        return {"out": out}
    w = x.sum(2)                                                         # rows, n_kv, length
    old = s["mass"][rows][:, :, :s["max_len"]]
    n = n[:, None, None]
    s["mass"][rows, :, :s["max_len"]] = torch.where(j < n - t, old + w, torch.where(j < n, w, old))
    return {"out": out, "mass": s["mass"]}


def _evict(s):
    c, rows = s["case"], s["rows"].long()
    page, n_kv, dev = c["page"], c["n_kv"], s["mass"].device
    n = s["lens"][rows].long()
    least = c["sinks"] + c["recent"]
    keep = s["budget"][rows].floor().long().clamp(min=least)
    goes = n > keep
    left = torch.where(goes, keep, n)
    s["dst_lens"].copy_(left)
    j = torch.arange(s["max_len"], device=dev)
    m = s["mass"][rows][:, :, :s["max_len"]]
    sure = (j < c["sinks"]) | ((j >= n[:, None] - c["recent"]) & (j < n[:, None]))
    m = torch.where(sure[:, None], math.inf, m)
    m = torch.where((j < n[:, None])[:, None], m, -math.inf)
    by = torch.sort(m, dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(by).scatter_(-1, by, j.expand_as(by))
    stays = (rank < left[:, None, None]) & goes[:, None, None]
    b, h, src = stays.nonzero(as_tuple=True)                             # in the tokens' order
    to = stays.cumsum(-1)[b, h, src] - 1
    s["kept"][b, h, to] = src.to(torch.int32)
    old = s["table"][rows].long()[b, src // page], src % page, h
    new = s["dst_table"].long()[b, to // page], to % page, h
    for name in ("k", "v"):
        whole = torch.uint8 if c["kv"] == "e4m3" else torch.int16
        s["dst_" + name].view(whole)[new] = s[name].view(whole)[old]
    s["mass_out"][rows[b], h, to] = s["mass"][rows[b], h, src]
    return {"k": _values(s["dst_k"]), "v": _values(s["dst_v"]), "len": s["dst_lens"], "kept": s["kept"], "mass": s["mass_out"]}


def _verify(s):
    c, dev = s["case"], s["target"].device
    rows, n, vocab = c["rows"], c["drafts"], c["vocab"]
    i = torch.arange(rows, device=dev)
    t = torch.arange(n, device=dev)
    x = s["tokens"].long()
    p = s["target"][i[:, None], t[None], x].double()
    q = s["draft"][i[:, None], t[None], x].double() if c["dist"] else torch.ones_like(p)
    ok = (s["u"].double() * q < p) & (t < s["n_draft"][:, None])
    a = ok.long().cumprod(1).sum(1)                                      # accepted drafts
    w = s["target"][i, a].double()
    rejected = (a < s["n_draft"])[:, None]
    if n:
        at = a.clamp(max=n - 1)
        minus = s["draft"][i, at].double() if c["dist"] else torch.zeros_like(w).scatter(1, x[i, at][:, None], math.inf)
        rest = (w - minus).clamp(min=0)
        w = torch.where(rejected & (rest.sum(1, keepdim=True) > 0), rest, w)
    total = w.cumsum(1)
    over = total > s["u_sample"].double()[:, None] * total[:, -1:]
    last = torch.where(w > 0, torch.arange(vocab, device=dev), -1).amax(1)
    pick = torch.where(over.any(1), over.int().argmax(1), last)
    col = torch.arange(n + 1, device=dev)
    wide = torch.cat([x, x.new_zeros(rows, 1)], 1)
    out = torch.where(col < a[:, None], wide, torch.where(col == a[:, None], pick[:, None], -1)).to(torch.int32)
    emitted = (a + 1).to(torch.int32)
    r = s["rows"].long()
    s["observed"].index_add_(0, r, emitted)
    s["lens"][r] = (s["lens"][r] - (s["n_draft"] - a)).clamp(min=0).to(torch.int32)
    return {"tokens": out, "emitted": emitted, "observed": s["observed"], "lens": s["lens"]}


# ---- work and 64-bit values -------------------------------------------------------

def _size(kind):
    return {"f32": 4, "f16": 2, "bf16": 2, "e4m3": 1}[kind]


def work(case):
    if case["op"] == "attention":
        tokens = case["hi"] + (case["rows"] - 1) * (case["lo"] + case["hi"]) / 2
        if case["window"]:
            tokens = min(tokens, case["rows"] * (case["window"] + case["tokens"] + case["sinks"]))
        heads = case["n_kv"] * case["group"] * case["tokens"]
        b = tokens * case["n_kv"] * 2 * case["dim"] * _size(case["kv"]) + 2 * case["rows"] * heads * case["dim"] * _size(case["q"])
        if case["mass"]:
            b += 8 * tokens * case["n_kv"]
        return {"bytes": b, "flops": 4 * tokens * heads * case["dim"]}
    if case["op"] == "evict":
        tokens = case["hi"] + (case["rows"] - 1) * (case["lo"] + case["hi"]) / 2
        lo, hi = case["keep_lo"], case["keep_hi"]
        # share kept of the requests that are cut: the budgets' share is uniform, cut below 1
        kept = (min(hi, 1) ** 2 - lo ** 2) / 2 / (hi - lo) if hi > lo else lo
        cut = min(1, (1 - lo) / (hi - lo)) if hi > lo else 1
        b = case["n_kv"] * tokens * (4 * cut + kept * (4 * case["dim"] * _size(case["kv"]) + 8))
        return {"bytes": b, "flops": 0}
    rows, n = case["rows"], max(0, case["drafts"] - 1)
    e = _size(case["type"])
    rejected = 1 - ACCEPT ** n
    b = rows * (case["vocab"] * e * (1 + (rejected if case["dist"] else 0)) + 2 * case["drafts"] * (e + 4) + 40)
    return {"bytes": b, "flops": 2 * rows * case["vocab"]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(s)
    if case["op"] == "evict":
        return _exact_evict(s)
    return _exact_verify(s)


def _exact_attention(s):
    """Request by request and head by head, from the definition."""
    c = s["case"]
    t, group, page = c["tokens"], c["group"], c["page"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    mass = s["mass"].double() if c["mass"] else None
    for i, r in enumerate(s["rows"].tolist()):
        n = int(s["lens"][r])
        pos = torch.arange(n, device="cuda")
        pages = s["table"][r].long()[pos // page]
        for h in range(c["n_kv"]):
            k = s["k"][pages, pos % page, h].double()
            v = s["v"][pages, pos % page, h].double()
            if "k_scale" in s:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            summed = torch.zeros(n, dtype=torch.float64, device="cuda")
            for b in range(t):
                p = n - t + b
                if p < 0:
                    continue
                see = torch.nonzero((pos <= p) & ((pos > p - c["window"]) | (pos < c["sinks"])) if c["window"] else pos <= p)[:, 0]
                q = s["q"][i, b, h * group:(h + 1) * group].double()
                w = torch.softmax((q @ k[see].T) / math.sqrt(c["dim"]), -1)
                out[i, b, h * group:(h + 1) * group] = w @ v[see]
                summed[see] += w.sum(0)
            if mass is not None:
                mass[r, h, :n] = torch.where(pos < n - t, mass[r, h, :n] + summed, summed)
    return {"out": out, "mass": mass} if c["mass"] else {"out": out}


def _exact_evict(s):
    """Which tokens stay, request by request and head by head; the copies are
    the inputs' own values."""
    c, page = s["case"], s["case"]["page"]
    k, v, mass = s["dst_k"].double(), s["dst_v"].double(), s["mass_out"].double()
    lens, kept = s["dst_lens"].clone(), s["kept"].clone()
    for i, r in enumerate(s["rows"].tolist()):
        n = int(s["lens"][r])
        keep = max(int(math.floor(float(s["budget"][r]))), c["sinks"] + c["recent"])
        lens[i] = min(n, keep)
        if n <= keep:
            continue
        lo, hi = c["sinks"], n - c["recent"]
        for h in range(c["n_kv"]):
            m = s["mass"][r, h, :n].double()
            by = torch.sort(-m[lo:hi], stable=True).indices[:keep - c["sinks"] - c["recent"]] + lo
            every = torch.arange(n, device="cuda")
            idx = torch.cat([every[:lo], by.sort().values, every[hi:]])
            to = torch.arange(keep, device="cuda")
            pages, new = s["table"][r].long()[idx // page], s["dst_table"][i].long()[to // page]
            k[new, to % page, h] = s["k"][pages, idx % page, h].double()
            v[new, to % page, h] = s["v"][pages, idx % page, h].double()
            mass[r, h, :keep] = m[idx]
            kept[i, h, :keep] = idx.to(torch.int32)
    return {"k": k, "v": v, "len": lens, "kept": kept, "mass": mass}


def _exact_verify(s):
    """Token by token, from the definition."""
    c = s["case"]
    out = torch.full((c["rows"], c["drafts"] + 1), -1, dtype=torch.int32)
    emitted = torch.zeros(c["rows"], dtype=torch.int32)
    observed, lens = s["observed"].cpu(), s["lens"].cpu()
    n_draft, tokens, u = s["n_draft"].tolist(), s["tokens"].tolist(), s["u"].tolist()
    for i, r in enumerate(s["rows"].tolist()):
        a = 0
        while a < n_draft[i]:
            x = tokens[i][a]
            if not u[i][a] * (float(s["draft"][i, a, x]) if c["dist"] else 1.0) < float(s["target"][i, a, x]):
                break
            out[i, a] = x
            a += 1
        w = s["target"][i, a].double()
        if a < n_draft[i]:
            rest = w.clone()
            if c["dist"]:
                rest = torch.clamp(w - s["draft"][i, a].double(), min=0)
            else:
                rest[tokens[i][a]] = 0
            w = rest if float(rest.sum()) > 0 else w
        sums = w.cumsum(0)
        out[i, a] = int(torch.searchsorted(sums, s["u_sample"][i].double() * sums[-1], right=True))
        emitted[i] = a + 1
        observed[r] += a + 1
        lens[r] = max(0, int(lens[r]) - (n_draft[i] - a))
    return {"tokens": out, "emitted": emitted, "observed": observed, "lens": lens}
