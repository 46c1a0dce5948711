"""Cases of the decoding and scoring operators: a 4-bit key/value cache (append and read
back), attention over it, eviction by accumulated attention weight, and log probabilities of
given tokens with their gradient.

`own` False computes an operator in plain torch operations in 32 bits; `own` True makes the
calls of the framework's binding. Both read the same state. The cache holds, per page and
key/value head, granules of 16 tokens: 16 rows of 4-bit key codes (head dim / 2 bytes; dim 2j
in the low half of byte j), 16 rows of value codes, then 16 (scale, offset) bf16 pairs of the
keys and 16 of the values; a value is scale * code + offset.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decoded token of 16 sequences enters the cache: a call whose latency counts
        {"name": "append-step", "op": "append", "batch": 16, "tokens": 1, "ragged": False, "kv_heads": 8, "dim": 128,
         "page": 64, "dtype": "bf16", "past": 1500},
        # packed prompts of different lengths enter an empty cache, as after a prompt's forward pass
        {"name": "append-prompts", "op": "append", "batch": 40, "tokens": 2048, "ragged": True, "kv_heads": 8,
         "dim": 128, "page": 64, "dtype": "bf16", "past": 0},
        # one token of one sequence over a short cache: the latency of interactive decoding
        {"name": "attend-one", "op": "attend", "batch": 1, "len": 1025, "queries": 1, "heads": 32, "kv_heads": 8,
         "dim": 128, "page": 64, "dtype": "bf16", "track": False, "empty": False},
        # ordinary serving: 64 sequences of different lengths, one token each, eight heads to a cache head
        {"name": "attend-batch", "op": "attend", "batch": 64, "len": 8192, "queries": 1, "heads": 64, "kv_heads": 8,
         "dim": 128, "page": 64, "dtype": "bf16", "track": False, "empty": False},
        # long documents, with the attention weight of every cached token accumulated for a later eviction
        {"name": "attend-long", "op": "attend", "batch": 16, "len": 131072, "queries": 1, "heads": 64, "kv_heads": 8,
         "dim": 128, "page": 128, "dtype": "bf16", "track": True, "empty": False},
        # drafted tokens are verified: one to eight queries a sequence, one sequence still empty, 32-bit activations
        {"name": "attend-draft", "op": "attend", "batch": 24, "len": 4099, "queries": 8, "heads": 32, "kv_heads": 8,
         "dim": 64, "page": 16, "dtype": "f32", "track": True, "empty": True},
        # a running cache goes 64 tokens over its budget and is cut back, as every 64 steps of decoding
        {"name": "evict-step", "op": "evict", "batch": 32, "len": 4160, "budget": 4096, "recent": 256, "sink": 4,
         "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "ragged": False},
        # long prompts are cut to a fixed budget once, lengths differing
        {"name": "evict-prompt", "op": "evict", "batch": 8, "len": 32771, "budget": 4096, "recent": 512, "sink": 4,
         "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "ragged": True},
        # the tokens that a small batch has just sampled are scored, with five alternatives
        {"name": "score-step", "op": "score", "rows": 8, "vocab": 128000, "top": 5, "dtype": "bf16", "masked": False},
        # perplexity of a text with twenty alternatives a token
        {"name": "score-corpus", "op": "score", "rows": 4096, "vocab": 128000, "top": 20, "dtype": "bf16",
         "masked": False},
        # the gradient of a few rows of a small vocabulary of odd size, entropy term included, some logits masked
        {"name": "grad-few", "op": "grad", "rows": 96, "vocab": 32001, "dtype": "f32", "masked": True, "entropy": True},
        # the loss gradient that calibration starts its backward pass from
        {"name": "grad-corpus", "op": "grad", "rows": 4096, "vocab": 128000, "dtype": "bf16", "masked": False,
         "entropy": False},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "attend", "attend", "evict", "score", "grad"])
    dtype = rng.choice(["bf16", "f32"])
    if op in ("score", "grad"):
        vocab = log(1000, 200000)
        rows = log(1, max(1, min(8192, 250_000_000 // vocab)))
        c = {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "masked": rng.random() < 0.3}
        c.update({"top": rng.choice([0, 1, 5, 20, 32])} if op == "score" else {"entropy": rng.random() < 0.5})
        return c
    dim, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128, 256])
    kv = rng.choice([1, 2, 4, 8, 8])
    if op == "append":
        batch = log(1, 128)
        return {"op": op, "batch": batch, "tokens": log(1, max(1, 65536 // batch)), "ragged": rng.random() < 0.7,
                "kv_heads": kv, "dim": dim, "page": page, "dtype": dtype, "past": rng.choice([0, 1, log(1, 4096)])}
    if op == "attend":
        batch = log(1, 128)
        most = max(1, min(131072, 8_000_000 // (batch * kv)))
        queries = rng.choice([1, 1, 1, 2, 5, 8])
        return {"op": op, "batch": batch, "len": log(1, most), "queries": queries,
                "heads": kv * rng.choice([1, 2, 4, 7, 8, 8, 16]), "kv_heads": kv, "dim": dim, "page": page, "dtype": dtype,
                "track": rng.random() < 0.4, "empty": rng.random() < 0.2}
    batch = log(1, 64)
    length = log(64, max(64, min(131072, 2_000_000 // (batch * kv))))
    budget = max(16, int(length * rng.choice([0.1, 0.3, 0.7, 0.98])))
    return {"op": op, "batch": batch, "len": length, "budget": budget, "recent": budget // rng.choice([2, 4, 16]),
            "sink": rng.choice([0, 1, 4]), "kv_heads": kv, "dim": dim, "page": page, "dtype": dtype,
            "ragged": rng.random() < 0.5}


# ----------------------------------------------------------------------------- inputs
def _lengths(g, batch, most, ragged):
    """Lengths on the host: `most`, or spread between a quarter of it and it, the longest `most`, in an order of the seed's."""
    if not ragged:
        return [most] * batch
    spread = [max(1, int(most * (0.25 + 0.75 * (0.618034 * i % 1)))) for i in range(1, batch)] + [most]
    return [spread[i] for i in torch.randperm(batch, generator=g).tolist()]


def _starts(counts, dev):
    return torch.tensor([0] + counts, dtype=torch.int64).cumsum(0).to(device=dev, dtype=torch.int32)


def _keys(n, heads, dim, g, dev):
    """Keys or values as they come from a projection: normal, a few channels of a head several times the rest."""
    chan = torch.exp(0.4 * torch.randn(heads, dim, device=dev, generator=g))
    chan[:, :: max(1, dim // 3)] *= 4
    return torch.randn(n, heads, dim, device=dev, generator=g) * chan


def _pool(case, g, dev):
    """A pool of pages in an order of its own, filled with quantized keys and values, and each sequence's table."""
    batch, heads, dim, page = case["batch"], case["kv_heads"], case["dim"], case["page"]
    slots = case["slots"]
    per = -(-slots // page)
    pages = batch * per + 3
    cache = torch.empty(pages, heads, page * (dim + 8), dtype=torch.uint8, device=dev)
    step = max(1, (1 << 26) // (heads * page * dim))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        k, v = (_pack(*_quantize(_keys(n * page, heads, dim, g, dev))) for _ in range(2))
        rows = [x.view(n, page // 16, 16, heads, -1).permute(0, 3, 1, 2, 4).reshape(n, heads, page // 16, -1)
                for x in (k[0], v[0], k[1], v[1])]
        cache[p:p + n] = torch.cat(rows, -1).view(n, heads, -1)
    order = torch.randperm(pages, device=dev, generator=g)[: batch * per]
    return cache, order.view(batch, per).to(torch.int32)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    h = torch.Generator().manual_seed(seed)
    op, dtype = case["op"], DTYPES[case["dtype"]]
    st = {"case": case}
    if op in ("score", "grad"):
        rows, vocab = case["rows"], case["vocab"]
        x = torch.randn(rows, vocab, device=dev, generator=g) * 2.5
        st["target"] = torch.randint(0, vocab, (rows,), device=dev, generator=g)
        # a confident model: the given token and some others stand out in most rows
        lift = torch.rand(rows, 1, device=dev, generator=g) * 14
        x.scatter_add_(1, st["target"][:, None], lift)
        x.scatter_add_(1, torch.randint(0, vocab, (rows, 8), device=dev, generator=g), 0.8 * lift.expand(rows, 8))
        if case["masked"]:  # tokens a grammar rules out, and a few positions that are not scored
            x[torch.rand(rows, vocab, device=dev, generator=g) < 0.2] = -math.inf
            x.scatter_(1, st["target"][:, None], lift)
            st["target"][torch.rand(rows, device=dev, generator=g) < 0.1] = -1
        st["logits"] = x.to(dtype)
        if op == "grad":
            st["g_logp"] = torch.randn(rows, device=dev, generator=g)
            st["g_entropy"] = torch.randn(rows, device=dev, generator=g) if case["entropy"] else None
            y = st["logits"].double() if rows * vocab < (1 << 28) else st["logits"].float()
            st["lse"] = torch.logsumexp(y, 1).float()
            lp = y - st["lse"].to(y.dtype)[:, None]
            st["entropy"] = -(lp.exp() * torch.where(lp > -math.inf, lp, 0.0)).sum(1).float()
            st["grad"] = torch.empty_like(st["logits"])
        return st
    batch, heads, dim = case["batch"], case["kv_heads"], case["dim"]
    if op == "append":
        counts = _lengths(h, batch, case["tokens"], case["ragged"])
        st["lens"] = torch.full((batch,), case["past"], dtype=torch.int32, device=dev)
        st["seen"] = st["lens"] + 7  # seven tokens of each sequence were evicted before
        st["start"], total = _starts(counts, dev), sum(counts)
        slots = case["past"] + case["tokens"]
        st["cache"], st["table"] = _pool({**case, "slots": slots}, g, dev)
        st["k"], st["v"] = (_keys(total, heads, dim, g, dev).to(dtype) for _ in range(2))
        st["acc"] = torch.full((batch, heads, slots), 0.5, device=dev)
        st["pos"] = torch.full((batch, heads, slots), -1, dtype=torch.int32, device=dev)
        return st
    if op == "attend":
        st["lens"] = torch.tensor(_lengths(h, batch, case["len"], batch > 1), dtype=torch.int32, device=dev)
        if case["empty"]:
            st["lens"][-1] = 0
        q = case["queries"]
        counts = [1 + i % q for i in torch.randperm(batch, generator=h).tolist()]
        st["start"], total = _starts(counts, dev), sum(counts)
        st["cache"], st["table"] = _pool({**case, "slots": case["len"]}, g, dev)
        # the queries come as a part of one projection's output: rows with a stride of their own
        wide = torch.randn(total, case["heads"] + 2 * heads, dim, device=dev, generator=g) * 1.2
        st["q"] = wide.to(dtype)[:, : case["heads"]]
        st["acc"] = torch.rand(batch, heads, case["len"], device=dev, generator=g) if case["track"] else None
        st["out"] = torch.empty(total, case["heads"], dim, dtype=dtype, device=dev)
        st["lse"] = torch.empty(total, case["heads"], device=dev)
        return st
    lens = _lengths(h, batch, case["len"], case["ragged"])
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    st["cache"], st["table"] = _pool({**case, "slots": case["len"]}, g, dev)
    shape = (batch, heads, case["len"])
    # heavy hitters: a few tokens hold most of the weight, many round to the same small value
    st["acc"] = (torch.exp(3 * torch.randn(shape, device=dev, generator=g)) * 256).round() / 256
    # a part of each cache is in the order of an earlier eviction: positions permuted, each once
    pos = torch.arange(case["len"], device=dev).expand(shape).clone()
    half = min(lens) // 2
    pos[..., :half] = torch.argsort(torch.rand((batch, heads, half), device=dev, generator=g), dim=-1)
    st["pos"] = pos.to(torch.int32)
    st["seen"] = st["lens"].clone()
    st["acc_out"], st["pos_out"] = torch.zeros(shape, device=dev), torch.zeros(shape, dtype=torch.int32, device=dev)
    st["lens_out"] = torch.zeros_like(st["lens"])
    st["start"] = (torch.arange(batch + 1, device=dev) * case["budget"]).to(torch.int32)
    st["first"] = torch.zeros_like(st["lens"])
    return st


# -------------------------------------------------------------------------- plain forms
def _quantize(x):
    """Codes (float), scale and offset of rows of 32-bit values: offset is the minimum rounded down to bf16, the
    scale a fifteenth of what is above it rounded up to bf16; a row with no finite range is NaN."""
    lo, hi = x.amin(-1), x.amax(-1)
    bits = lo.contiguous().view(torch.int32)
    off = ((bits + torch.where(bits < 0, 0xFFFF, 0).to(torch.int32)) & -65536).view(torch.float32)
    s = ((hi - off) / torch.full_like(hi, 15)).contiguous()  # by a number, the quotient would be a product with 1 / 15
    s = ((s.view(torch.int32) + 0xFFFF) & -65536).view(torch.float32)
    bad = ~(torch.isfinite(s) & torch.isfinite(off) & torch.isfinite(x).all(-1))
    s, off = torch.where(bad, math.nan, s), torch.where(bad, math.nan, off)
    c = torch.round((x - off[..., None]) / s[..., None]).clamp(0, 15)
    return torch.where((s > 0)[..., None], c, 0.0), s, off


def _pack(c, s, off):
    """(bytes of the codes [..., dim / 2], bytes of scale and offset [..., 4])."""
    c = c.to(torch.uint8)
    param = torch.stack([s, off], -1).to(torch.bfloat16).view(torch.uint8)
    return c[..., ::2] | (c[..., 1::2] << 4), param


def _value(codes, param):
    """The 32-bit values of rows of packed codes [..., dim / 2] with their parameters' bytes [..., 4]."""
    so = param.contiguous().view(torch.bfloat16).float()
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() * so[..., :1] + so[..., 1:]


def _unpack(block, dim):
    """Keys and values in 32 bits, [..., tokens, dim], from blocks [..., page * (dim + 8)] of a page and head."""
    row = block.reshape(*block.shape[:-1], -1, 16 * (dim + 8))
    cut = [8 * dim, 8 * dim, 64, 64]
    parts = torch.split(row, cut, -1)
    return [_value(c.unflatten(-1, (16, -1)), p.unflatten(-1, (16, -1))).flatten(-3, -2) for c, p in zip(parts[:2], parts[2:])]


def _dense(st, dim):
    """Keys and values of every sequence, [batch, kv heads, slots, dim] in 32 bits."""
    block = st["cache"][st["table"].long()]  # [batch, pages of a sequence, heads, bytes]
    return [x.transpose(1, 2).flatten(2, 3) for x in _unpack(block, dim)]


def _plain_append(st):
    c = st["case"]
    heads, dim, page = c["kv_heads"], c["dim"], c["page"]
    start, lens = st["start"].long(), st["lens"].long()
    total = st["k"].shape[0]
    i = torch.arange(total, device=start.device)
    b = torch.searchsorted(start, i, right=True) - 1
    slot = lens[b] + i - start[b]
    at = st["table"].long()[b, slot // page]
    off = slot % page
    gran = st["cache"].view(st["cache"].shape[0], heads, page // 16, 16 * (dim + 8))
    widths = (dim // 2, dim // 2, 4, 4)
    rows = [x.unflatten(-1, (16, w)) for x, w in zip(torch.split(gran, [16 * w for w in widths], -1), widths)]
    k, v = (_pack(*_quantize(st[n].float())) for n in ("k", "v"))
    for row, part in zip(rows, (k[0], v[0], k[1], v[1])):
        row[at, :, off // 16, off % 16] = part
    st["acc"][b, :, slot] = 0.0
    st["pos"][b, :, slot] = (st["seen"].long()[b] + i - start[b]).to(torch.int32)[:, None]
    counts = (start[1:] - start[:-1]).to(torch.int32)
    # read back, as the values that the codes stand for
    held = [row[at, :, off // 16, off % 16] for row in rows]
    k, v = (_value(c, p).to(st["k"].dtype) for c, p in (held[::2], held[1::2]))
    return {"k": k, "v": v, "lens": st["lens"] + counts, "seen": st["seen"] + counts, "acc": st["acc"], "pos": st["pos"]}


def _plain_attend(st):
    c = st["case"]
    kv, dim, q = c["kv_heads"], c["dim"], c["queries"]
    group = c["heads"] // kv
    k, v = _dense(st, dim)
    batch, slots = k.shape[0], k.shape[2]
    start, lens = st["start"].long(), st["lens"].long()
    count = start[1:] - start[:-1]
    i = torch.arange(q, device=start.device)
    real = i < count[:, None]
    at = torch.where(real, start[:-1, None] + i, 0)
    rows = st["q"].float()[at].view(batch, q, kv, group, dim).permute(0, 2, 1, 3, 4).reshape(batch, kv, -1, dim)
    s = torch.matmul(rows, k.transpose(2, 3)) / math.sqrt(dim)
    # query i of n sees the slots up to the length less the n - 1 - i tokens after it
    most = (lens[:, None] - (count[:, None] - 1 - i)).repeat_interleave(group, 1)
    seen = torch.arange(slots, device=start.device) < most[:, None, :, None]
    s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(s - torch.where(m > -math.inf, m, 0.0)), 0.0)
    z = p.sum(-1, keepdim=True)
    p = torch.where(z > 0, p / z, 0.0)
    lse = (m + torch.log(z))[..., 0]
    o = torch.matmul(p, torch.where((torch.arange(slots, device=v.device) < lens[:, None])[:, None, :, None], v, 0.0))

    def packed(x):
        x = x.view(batch, kv, q, group, -1).permute(0, 2, 1, 3, 4).reshape(batch, q, kv * group, -1)
        return x[real]

    st["out"].copy_(packed(o))
    st["lse"].copy_(packed(lse[..., None])[..., 0])
    got = {"out": st["out"], "lse": st["lse"]}
    if c["track"]:
        weight = p * real.repeat_interleave(group, 1)[:, None, :, None]
        st["acc"] += weight.sum(2)[..., : st["acc"].shape[2]]
        got["acc"] = st["acc"]
    return got


def _plain_evict(st):
    c = st["case"]
    kv, dim, budget, page = c["kv_heads"], c["dim"], c["budget"], c["page"]
    batch, _, slots = st["acc"].shape
    dev = st["acc"].device
    lens, j = st["lens"].long()[:, None, None], torch.arange(slots, device=dev)
    pos = st["pos"].long()
    safe = (pos >= st["seen"].long()[:, None, None] - c["recent"]) | (pos < c["sink"])
    key = torch.where(safe, math.inf, st["acc"])
    key = torch.where(j < lens, key, -math.inf)
    rank = torch.argsort(key, dim=-1, descending=True, stable=True)
    keep = torch.zeros_like(key, dtype=torch.bool).scatter_(-1, rank[..., :budget], True) & (j < lens)
    # the kept slots past the budget, in order, fill the free slots before it, in order
    front = min(budget, slots)
    place = torch.arange(slots, device=dev).expand(key.shape).clone()
    hole = ~keep & (j < budget) & (j < lens)
    tail = keep & (j >= budget)
    n = torch.cumsum(tail.long(), -1) - 1
    src = torch.full((batch, kv, slots + 1), 0, dtype=torch.long, device=dev)
    src.scatter_(-1, torch.where(tail, n, slots), place)
    fill = torch.cumsum(hole.long(), -1) - 1
    place = torch.where(hole, src.gather(-1, fill.clamp(min=0)), place)[..., :front]
    new = torch.minimum(st["lens"], torch.full_like(st["lens"], budget))
    live = j[:front] < new[:, None, None]
    st["acc_out"][..., :front] = torch.where(live, st["acc"].gather(-1, place), st["acc_out"][..., :front])
    st["pos_out"][..., :front] = torch.where(live, st["pos"].gather(-1, place), st["pos_out"][..., :front])
    st["lens_out"].copy_(new)
    # move the packed rows
    gran = st["cache"].view(-1, kv, page // 16, 16 * (dim + 8))
    b, h = torch.arange(batch, device=dev)[:, None, None], torch.arange(kv, device=dev)[:, None]
    to = j[:front].expand(place.shape)
    t = st["table"].long()
    base = 0
    for w in (dim // 2, dim // 2, 4, 4):
        rows = gran[..., base:base + 16 * w].unflatten(-1, (16, w))
        moved = rows[t[b, place // page], h, place % page // 16, place % 16]
        rows[t[b, to // page], h, to % page // 16, to % 16] = moved
        base += 16 * w
    k, v = _dense(st, dim)
    dtype = DTYPES[c["dtype"]]

    def kept(x):
        x = torch.where(live[..., None], x[:, :, :front], 0.0)
        x = torch.nn.functional.pad(x, (0, 0, 0, budget - front))
        return x.transpose(1, 2).flatten(0, 1).to(dtype)

    return {"k": kept(k), "v": kept(v), "acc": st["acc_out"], "pos": st["pos_out"], "lens": st["lens_out"]}


def _plain_score(st):
    k = st["case"]["top"]
    x = st["logits"].float()
    rows, vocab = x.shape
    m = x.amax(1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    z = e.sum(1, keepdim=True)
    log_z = torch.log(z)
    lse = (m + log_z)[:, 0]
    entropy = log_z[:, 0] - (e * torch.where(d > -math.inf, d, 0.0)).sum(1) / z[:, 0]
    y = st["target"]
    logp = torch.where(y >= 0, d.gather(1, y.clamp(min=0)[:, None])[:, 0] - log_z[:, 0], 0.0)
    got = {"logp": logp, "entropy": entropy, "lse": lse}
    del e
    if k:
        # an order-preserving whole number of the value above the one of the token: no ties left
        bits = x.view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 20) + (vocab - 1 - torch.arange(vocab, device=x.device))
        del bits
        top = torch.topk(key, k, 1).values
        ids = vocab - 1 - (top & ((1 << 20) - 1))
        got["top_id"] = ids.to(torch.int32)
        got["top_logp"] = d.gather(1, ids) - log_z
    return got


def _plain_grad(st):
    x = st["logits"].float()
    lp = x - st["lse"][:, None]
    p = torch.exp(lp)
    y = st["target"]
    g = torch.where(y >= 0, st["g_logp"], 0.0)
    d = -g[:, None] * p
    d.scatter_add_(1, y.clamp(min=0)[:, None], g[:, None])
    if st["g_entropy"] is not None:
        d -= st["g_entropy"][:, None] * p * (torch.where(p > 0, lp, 0.0) + st["entropy"][:, None])
    st["grad"].copy_(d)
    return {"grad": st["grad"]}


# ------------------------------------------------------------------- the framework's calls
def _kept(st, name, make):
    if name not in st:
        st[name] = make()
    return st[name]


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def _own_append(kq, st):
    lens = _kept(st, "lens_out", lambda: torch.empty_like(st["lens"]))
    seen = _kept(st, "seen_out", lambda: torch.empty_like(st["seen"]))
    k = _kept(st, "k_out", lambda: torch.empty_like(st["k"]))
    v = _kept(st, "v_out", lambda: torch.empty_like(st["v"]))
    kq.kq_kv_append(st["k"], st["v"], st["start"], st["lens"], st["cache"], st["table"], lens_out=lens, acc=st["acc"],
                    pos=st["pos"], seen=st["seen"], seen_out=seen)
    kq.kq_kv_read(st["cache"], st["table"], st["start"], st["lens"], lens, k, v)
    return {"k": k, "v": v, "lens": lens, "seen": seen, "acc": st["acc"], "pos": st["pos"]}


def _own_attend(kq, st):
    ws = _kept(st, "ws", lambda: _bytes(kq.kq_kv_attend_workspace(st["q"], st["cache"], st["table"], st["acc"])))
    kq.kq_kv_attend(st["q"], st["start"], st["lens"], st["cache"], st["table"], st["out"], ws,
                    scale=1 / math.sqrt(st["case"]["dim"]), lse=st["lse"], acc=st["acc"])
    got = {"out": st["out"], "lse": st["lse"]}
    if st["acc"] is not None:
        got["acc"] = st["acc"]
    return got


def _own_evict(kq, st):
    c = st["case"]
    ws = _kept(st, "ws", lambda: _bytes(kq.kq_kv_evict_workspace(st["acc"], c["budget"])))
    rows = (c["batch"] * c["budget"], c["kv_heads"], c["dim"])
    k, v = (_kept(st, n, lambda: torch.empty(rows, dtype=DTYPES[c["dtype"]], device="cuda")) for n in ("k_out", "v_out"))
    kq.kq_kv_evict(st["cache"], st["table"], st["lens"], st["acc"], st["pos"], st["seen"], c["dim"], c["budget"],
                   c["recent"], c["sink"], st["lens_out"], st["acc_out"], st["pos_out"], ws)
    kq.kq_kv_read(st["cache"], st["table"], st["start"], st["first"], st["lens_out"], k, v)
    return {"k": k, "v": v, "acc": st["acc_out"], "pos": st["pos_out"], "lens": st["lens_out"]}


def _own_score(kq, st):
    rows, k = st["case"]["rows"], st["case"]["top"]

    def make():
        f = [torch.empty(rows, device="cuda") for _ in range(3)]
        return f + [torch.empty(rows, k, dtype=torch.int32, device="cuda"), torch.empty(rows, k, device="cuda")]

    logp, entropy, lse, top_id, top_logp = _kept(st, "results", make)
    kq.kq_token_logprobs(st["logits"], st["target"], logp, entropy=entropy, lse=lse, top_id=top_id if k else None,
                         top_logp=top_logp if k else None)
    got = {"logp": logp, "entropy": entropy, "lse": lse}
    return {**got, "top_id": top_id, "top_logp": top_logp} if k else got


def _own_grad(kq, st):
    kq.kq_token_logprobs_grad(st["logits"], st["target"], st["lse"], st["g_logp"], st["grad"], entropy=st["entropy"],
                              g_entropy=st["g_entropy"])
    return {"grad": st["grad"]}


def run(state):
    if own:
        from paper_2607_07964_gb300 import kronq as kq
        return {"append": _own_append, "attend": _own_attend, "evict": _own_evict, "score": _own_score,
                "grad": _own_grad}[state["case"]["op"]](kq, state)
    return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict, "score": _plain_score,
            "grad": _plain_grad}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------- work
def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    size = 2 if case["dtype"] == "bf16" else 4
    op = case["op"]
    if op == "score":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * size + case["rows"] * (20 + 8 * case["top"]), "flops": 6 * n}
    if op == "grad":
        n = case["rows"] * case["vocab"]
        return {"bytes": 2 * n * size + 24 * case["rows"], "flops": (9 if case["entropy"] else 4) * n}
    heads, dim, batch = case["kv_heads"], case["dim"], case["batch"]
    token = dim + 8  # a cached token of a head: two rows of codes and their parameters
    mean = 0.625 * batch + 0.375 if batch > 1 else 1.0  # expected lengths, in the longest one's
    if op == "append":
        n = heads * case["tokens"] * (mean if case["ragged"] else batch)
        # tokens in, codes and position and weight out; the codes in again, values out
        return {"bytes": n * (2 * 2 * dim * size + 2 * token + 8), "flops": 12 * n * dim}
    if op == "attend":
        cached = heads * case["len"] * (mean if batch > 1 else 1)
        rows = batch * (1 if case["queries"] == 1 else (case["queries"] + 1) / 2)
        per = rows / batch * case["heads"] / heads
        return {"bytes": cached * (token + (8 if case["track"] else 0)) + rows * case["heads"] * (2 * dim * size + 4),
                "flops": 4 * cached * per * dim}
    n = heads * case["len"] * (mean if case["ragged"] else batch)
    kept = min(n, heads * batch * case["budget"])
    moved = kept * (1 - kept / n)
    return {"bytes": 8 * n + 8 * kept + 2 * moved * token + kept * (token + 2 * dim * size), "flops": 4 * n + 4 * kept * dim}


# ------------------------------------------------------------------- 64 bits, written apart
def _values64(cache, table, page, dim):
    """The cache's keys and values in 64 bits, [batch, heads, slots, dim], token by token from the bytes' places."""
    slots = table.shape[1] * page
    t = torch.arange(slots, device=cache.device)
    byte = torch.arange(dim, device=cache.device) // 2
    shift = (torch.arange(dim, device=cache.device) % 2) * 4
    flat = cache.view(cache.shape[0], cache.shape[1], -1)
    at = (t % page // 16) * 16 * (dim + 8)
    got = []
    for which in range(2):
        codes = at[:, None] + which * 8 * dim + (t % 16)[:, None] * (dim // 2) + byte
        param = at[:, None] + 16 * dim + which * 64 + (t % 16)[:, None] * 4 + torch.arange(4, device=cache.device)
        val = []
        for b in range(table.shape[0]):
            own_pages = flat[table[b].long()].transpose(0, 1)  # [heads, pages, bytes]
            p = (t // page)[:, None]
            c = (own_pages[:, p, codes].to(torch.int32) >> shift & 15).double()
            w = own_pages[:, p, param].to(torch.int32)
            so = torch.stack([w[..., 0] | w[..., 1] << 8, w[..., 2] | w[..., 3] << 8], -1) << 16
            so = so.to(torch.int32).view(torch.float32).double()
            val.append(c * so[..., :1] + so[..., 1:])
        got.append(val)
    return got


def _exact_append(st):
    c, got = st["case"], {}
    for n in ("k", "v"):
        x = st[n].double()
        lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)

        def coarse(y, up):  # y to 8 significant bits, upwards or downwards
            step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=1e-30))) - 7)
            return (torch.ceil(y / step) if up else torch.floor(y / step)) * step

        off = coarse(lo, False)
        s = coarse((hi - off) / 15, True)
        got[n] = off + s * torch.round((x - off) / s)
    counts = (st["start"][1:] - st["start"][:-1]).tolist()
    acc, pos = st["acc"], st["pos"]
    for b, n in enumerate(counts):
        acc[b, :, c["past"]:c["past"] + n] = 0
        pos[b, :, c["past"]:c["past"] + n] = torch.arange(n, device=pos.device, dtype=pos.dtype) + st["seen"][b]
    more = torch.tensor(counts, dtype=torch.int32, device=pos.device)
    return {**got, "lens": st["lens"] + more, "seen": st["seen"] + more, "acc": acc.double(), "pos": pos}


def _exact_attend(st):
    c = st["case"]
    group, dim = c["heads"] // c["kv_heads"], c["dim"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    acc = st["acc"].double() if c["track"] else None
    lens, start = st["lens"].tolist(), st["start"].tolist()
    for b, n in enumerate(lens):
        if not n:
            continue
        k, v = _values64(st["cache"], st["table"][b:b + 1], c["page"], dim)
        k, v = k[0][:, :n], v[0][:, :n]
        for i in range(start[b], start[b + 1]):
            see = n - (start[b + 1] - 1 - i)
            if see <= 0:
                continue
            q = st["q"][i].double().view(c["kv_heads"], group, dim)
            s = torch.einsum("hgd,hnd->hgn", q, k[:, :see]) / math.sqrt(dim)
            p = torch.softmax(s, -1)
            lse[i] = torch.logsumexp(s, -1).flatten()
            out[i] = torch.einsum("hgn,hnd->hgd", p, v[:, :see]).flatten(0, 1)
            if acc is not None:
                acc[b, :, :see] += p.sum(1)
    return {"out": out, "lse": lse, **({"acc": acc} if c["track"] else {})}


def _exact_evict(st):
    c = st["case"]
    heads, dim, budget = c["kv_heads"], c["dim"], c["budget"]
    n_b, slots = c["batch"], st["acc"].shape[2]
    k = torch.zeros(n_b, budget, heads, dim, dtype=torch.float64, device="cuda")
    v = torch.zeros_like(k)
    acc = torch.zeros(n_b, heads, slots, dtype=torch.float64)
    pos = torch.zeros(n_b, heads, slots, dtype=torch.int32)
    lens = st["lens"].tolist()
    weight, where = st["acc"].cpu().numpy(), st["pos"].cpu().numpy()
    for b, n in enumerate(lens):
        vals = _values64(st["cache"], st["table"][b:b + 1], c["page"], dim)
        for h in range(heads):
            held = list(range(min(n, budget)))
            if n > budget:
                safe = (where[b, h] >= n - c["recent"]) | (where[b, h] < c["sink"])
                prior = [(0, 0, j) if safe[j] else (1, -weight[b, h, j], j) for j in range(n)]
                chosen = {x[2] for x in sorted(prior)[:budget]}
                late = iter(sorted(j for j in chosen if j >= budget))
                held = [j if j in chosen else next(late) for j in range(budget)]
            at = torch.tensor(held, device="cuda")
            k[b, :len(held), h], v[b, :len(held), h] = vals[0][0][h, at], vals[1][0][h, at]
            acc[b, h, :len(held)] = torch.from_numpy(weight[b, h][held]).double()
            pos[b, h, :len(held)] = torch.from_numpy(where[b, h][held])
    return {"k": k.flatten(0, 1), "v": v.flatten(0, 1), "acc": acc, "pos": pos,
            "lens": torch.tensor([min(n, budget) for n in lens], dtype=torch.int32)}


def _exact_score(st):
    k = st["case"]["top"]
    rows, vocab = st["logits"].shape
    got = {"logp": [], "entropy": [], "lse": [], "top_id": [], "top_logp": []}
    step = max(1, (1 << 27) // vocab)
    for r in range(0, rows, step):
        x = st["logits"][r:r + step].double()
        lp = torch.log_softmax(x, 1)
        p = lp.exp()
        y = st["target"][r:r + step]
        got["lse"].append(torch.logsumexp(x, 1))
        got["entropy"].append(-torch.where(p > 0, p * lp, 0.0).sum(1))
        got["logp"].append(torch.where(y < 0, 0.0, lp[torch.arange(len(y), device=y.device), y.clamp(min=0)]))
        if k:
            best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
            got["top_id"].append(best.to(torch.int32))
            got["top_logp"].append(lp.gather(1, best))
    return {n: torch.cat(v) for n, v in got.items() if v}


def _exact_grad(st):
    rows, vocab = st["logits"].shape
    if rows * vocab > 600_000_000:
        return None
    grad = torch.empty(rows, vocab, dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // vocab)
    for r in range(0, rows, step):
        x = st["logits"][r:r + step].double()
        y = st["target"][r:r + step]
        lp = torch.log_softmax(x, 1)
        p = lp.exp()
        one = (torch.arange(vocab, device=y.device) == y[:, None]).double()
        d = st["g_logp"][r:r + step, None].double() * (one - p) * (y >= 0)[:, None]
        if st["g_entropy"] is not None:
            plp = torch.where(p > 0, p * lp, 0.0)
            d -= st["g_entropy"][r:r + step, None].double() * (plp - p * plp.sum(1, keepdim=True))
        grad[r:r + step] = d
    return {"grad": grad}


def exact(case, seed):
    if case["op"] == "evict" and case["batch"] * case["kv_heads"] * case["len"] > 4_000_000:
        return None
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "evict": _exact_evict, "score": _exact_score,
            "grad": _exact_grad}[case["op"]](st)
