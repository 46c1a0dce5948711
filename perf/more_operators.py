"""Cases of the operators around attention and at the end of a model: norm and rotation of queries and keys with
their gradient, attention over the 4-bit cache with a sliding window and first tokens that stay visible, and log
probabilities straight from hidden states (no logits kept) with their gradient.

`own` False computes an operator in plain torch operations in 32 bits; `own` True makes the calls of the framework's
binding. Both read the same state. Rotation frequencies are 64-bit fractions of a turn for one position, so that the
whole-number product with a position, which wraps at a turn, is exact. The cache holds, per page and key/value head,
granules of 16 tokens: 16 rows of 4-bit key codes (head dim / 2 bytes; dim 2j in the low half of byte j), 16 rows of
value codes, then 16 (scale, offset) bf16 pairs of the keys and 16 of the values; a value is scale * code + offset.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6  # of the norms


# ------------------------------------------------------------------------------- cases
def listed():
    return [
        # one decoded token of 16 sequences far into their texts: a call whose latency counts
        {"name": "rotate-step", "op": "rotate", "tokens": 16, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "far": 131072, "stretch": 1.0},
        # packed prompts of a batch
        {"name": "rotate-prompt", "op": "rotate", "tokens": 32768, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "far": 8192, "stretch": 1.0},
        # an odd number of tokens, a part of an unusual head, neighbours as pairs, frequencies stretched for a long text
        {"name": "rotate-part", "op": "rotate", "tokens": 4097, "heads": 28, "kv_heads": 4, "dim": 80, "rot": 32,
         "interleaved": True, "norm": False, "dtype": "f32", "far": 1000000, "stretch": 8.0},
        # the backward pass of calibration through the same place
        {"name": "rotate-grad", "op": "rotate_grad", "tokens": 16384, "heads": 32, "kv_heads": 8, "dim": 128, "rot": 128,
         "interleaved": False, "norm": True, "dtype": "bf16", "far": 2048, "stretch": 1.0},
        # one short text, few heads, a rotated part whose halves are no whole vectors
        {"name": "rotate-grad-odd", "op": "rotate_grad", "tokens": 777, "heads": 7, "kv_heads": 1, "dim": 64, "rot": 24,
         "interleaved": True, "norm": True, "dtype": "f32", "far": 777, "stretch": 1.0},
        # one token of one long text: the latency of interactive decoding
        {"name": "window-one", "op": "window", "batch": 1, "len": 131072, "window": 1024, "sink": 4, "queries": 1,
         "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "empty": False},
        # ordinary serving: 64 sequences, most of them far longer than the window
        {"name": "window-batch", "op": "window", "batch": 64, "len": 32768, "window": 4096, "sink": 4, "queries": 1,
         "heads": 64, "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "empty": False},
        # drafted tokens are verified: one to eight queries, an odd window, one sequence still empty, 32-bit activations
        {"name": "window-draft", "op": "window", "batch": 24, "len": 9001, "window": 515, "sink": 20, "queries": 8,
         "heads": 32, "kv_heads": 8, "dim": 64, "page": 16, "dtype": "f32", "empty": True},
        # the tokens that a small batch has just been given are scored
        {"name": "score-few", "op": "score", "rows": 8, "vocab": 128000, "hidden": 4096, "masked": False},
        # perplexity of a text
        {"name": "score-corpus", "op": "score", "rows": 4096, "vocab": 128000, "hidden": 4096, "masked": False},
        # a few rows of a small vocabulary of odd size, entropy term included, some positions not scored
        {"name": "grad-few", "op": "grad", "rows": 96, "vocab": 32001, "hidden": 1024, "masked": True, "entropy": True},
        # the loss gradient that calibration starts its backward pass from, with the head's own
        {"name": "grad-corpus", "op": "grad", "rows": 4096, "vocab": 128000, "hidden": 2048, "masked": False,
         "entropy": False},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotate", "rotate_grad", "window", "window", "score", "grad"])
    if op in ("score", "grad"):
        hidden, vocab = 8 * log(32, 1024), log(1000, 200000)
        vocab = min(vocab, 600_000_000 // hidden)
        most = (2_100_000_000_000 if op == "score" else 1_000_000_000_000) // (hidden * vocab)
        rows = log(1, max(1, min(8192, most, 520_000_000 // vocab)))
        c = {"op": op, "rows": rows, "vocab": vocab, "hidden": hidden, "masked": rng.random() < 0.4}
        return c if op == "score" else {**c, "entropy": rng.random() < 0.5}
    dtype, kv = rng.choice(["bf16", "f32"]), rng.choice([1, 2, 4, 8, 8])
    if op in ("rotate", "rotate_grad"):
        heads, dim = kv * rng.choice([1, 2, 4, 7, 8]), rng.choice([64, 80, 96, 128, 128, 256])
        rot = rng.choice([dim, dim, dim // 2, dim // 4, 2 * rng.randrange(1, dim // 2)])
        tokens = log(1, max(1, min(65536, (160_000_000 if op == "rotate" else 80_000_000) // ((heads + kv) * dim))))
        return {"op": op, "tokens": tokens, "heads": heads, "kv_heads": kv, "dim": dim, "rot": rot,
                "interleaved": rng.random() < 0.5, "norm": rng.random() < 0.6, "dtype": dtype,
                "far": log(tokens + 1, 2_000_000), "stretch": rng.choice([1.0, 1.0, 4.0, 32.0])}
    batch = log(1, 128)
    length = log(1, max(1, min(131072, 16_000_000 // (batch * kv))))
    return {"op": op, "batch": batch, "len": length, "window": log(1, 8192), "sink": rng.choice([0, 1, 4, 17, 64]),
            "queries": rng.choice([1, 1, 1, 2, 5, 8]), "heads": kv * rng.choice([1, 2, 4, 7, 8, 8, 16]), "kv_heads": kv,
            "dim": rng.choice([64, 128, 128]), "page": rng.choice([16, 32, 64, 128, 256]), "dtype": dtype,
            "empty": rng.random() < 0.2}


# ----------------------------------------------------------------------------- inputs
def _theta(case):
    """Radians for one position of each rotated pair, as a list of numbers. Stretched: waves that a text of 8192 holds
    less than once are slowed by the factor, those it holds four times or more are kept, those between in proportion."""
    n, got = case["rot"] // 2, []
    for j in range(n):
        t = 500000.0 ** (-j / n)
        keep = min(1.0, max(0.0, (8192 * t / (2 * math.pi) - 1) / 3))
        got.append(t * (keep + (1 - keep) / case["stretch"]))
    return got


def _length(case):
    """What a stretched rotation scales queries and keys by."""
    return 1.0 + 0.1 * math.log(case["stretch"])


def _lengths(g, batch, most, ragged):
    """Lengths on the host: `most`, or spread between a quarter of it and it, the longest `most`, in an order of the seed's."""
    if not ragged:
        return [most] * batch
    spread = [max(1, int(most * (0.25 + 0.75 * (0.618034 * i % 1)))) for i in range(1, batch)] + [most]
    return [spread[i] for i in torch.randperm(batch, generator=g).tolist()]


def _pool(case, g, dev):
    """A pool of pages in an order of its own, filled with quantized keys and values, and each sequence's table."""
    batch, heads, dim, page = case["batch"], case["kv_heads"], case["dim"], case["page"]
    per = -(-case["len"] // page)
    pages = batch * per + 3
    cache = torch.empty(pages, heads, page * (dim + 8), dtype=torch.uint8, device=dev)
    # codes of any value; scales and offsets as normal rows of channels of different sizes have them
    step = max(1, (1 << 27) // (heads * page * dim))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        codes = torch.randint(0, 256, (n, heads, page // 16, 16 * dim), dtype=torch.uint8, device=dev, generator=g)
        size = 0.2 * torch.exp(0.3 * torch.randn(n, heads, page // 16, 32, device=dev, generator=g))
        grid = torch.stack([size, -7.5 * size * (1 + 0.1 * torch.randn(size.shape, device=dev, generator=g))], -1)
        grid = grid.to(torch.bfloat16).view(torch.uint8).flatten(-2)
        cache[p:p + n] = torch.cat([codes, grid], -1).view(n, heads, -1)
    order = torch.randperm(pages, device=dev, generator=g)[: batch * per]
    return cache, order.view(batch, per).to(torch.int32)


def _prepare_rotate(case, st, g, dev):
    T, hq, hk, dim, dtype = case["tokens"], case["heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
    # queries and keys are parts of one projection's output: rows with a stride of their own
    wide = torch.randn(T, hq + 2 * hk, dim, device=dev, generator=g)
    wide *= torch.exp(0.4 * torch.randn(hq + 2 * hk, dim, device=dev, generator=g))
    wide = wide.to(dtype)
    st["q"], st["k"] = wide[:, :hq], wide[:, hq:hq + hk]
    # four texts one after the other, the last of them ending at the farthest position
    cut = -(-T // 4)
    i = torch.arange(T, device=dev)
    st["pos"] = (i % cut + (case["far"] - cut) * (i // cut) // 4).clamp(min=0).to(torch.int32)
    st["pos"][-1] = case["far"] - 1
    st["freq"] = torch.tensor([round(t / (2 * math.pi) * 2.0 ** 64) for t in _theta(case)], dtype=torch.int64, device=dev)
    st["wq"] = st["wk"] = None
    if case["norm"]:
        st["wq"], st["wk"] = ((1 + 0.2 * torch.randn(dim, device=dev, generator=g)).to(dtype) for _ in range(2))
    if case["op"] == "rotate_grad":
        st["gq"], st["gk"] = ((0.01 * torch.randn(T, h, dim, device=dev, generator=g)).to(dtype) for h in (hq, hk))
    st["q_out"], st["k_out"] = (torch.empty(T, h, dim, dtype=dtype, device=dev) for h in (hq, hk))


def _prepare_window(case, st, g, dev, h):
    batch, heads, dim = case["batch"], case["kv_heads"], case["dim"]
    st["lens"] = torch.tensor(_lengths(h, batch, case["len"], batch > 1), dtype=torch.int32, device=dev)
    if case["empty"]:
        st["lens"][-1] = 0
    counts = [1 + i % case["queries"] for i in torch.randperm(batch, generator=h).tolist()]
    total = sum(counts)
    st["start"] = torch.tensor([0] + counts).cumsum(0).to(device=dev, dtype=torch.int32)
    st["cache"], st["table"] = _pool(case, g, dev)
    wide = torch.randn(total, case["heads"] + 2 * heads, dim, device=dev, generator=g) * 1.2
    st["q"] = wide.to(DTYPES[case["dtype"]])[:, : case["heads"]]
    st["out"] = torch.empty(total, case["heads"], dim, dtype=DTYPES[case["dtype"]], device=dev)
    st["lse"] = torch.empty(total, case["heads"], device=dev)


def _prepare_score(case, st, g, dev):
    rows, vocab, hidden = case["rows"], case["vocab"], case["hidden"]
    w = torch.randn(vocab, hidden, device=dev, generator=g) * (2.5 / math.sqrt(hidden))
    st["w"] = w.to(torch.bfloat16)
    st["target"] = torch.randint(0, vocab, (rows,), device=dev, generator=g)
    # a confident model: hidden states lean towards their token's row, and towards another's
    lift = torch.rand(rows, 1, device=dev, generator=g) * 14
    other = torch.randint(0, vocab, (rows,), device=dev, generator=g)
    x = torch.randn(rows, hidden, device=dev, generator=g)
    x += lift / 6.25 * (w[st["target"]] + 0.8 * w[other])
    st["x"] = x.to(torch.bfloat16)
    del w, x
    if case["masked"]:  # positions that are not scored
        st["target"][torch.rand(rows, device=dev, generator=g) < 0.1] = -1
    if case["op"] == "grad":
        st["g_logp"] = torch.randn(rows, device=dev, generator=g)
        st["g_entropy"] = torch.randn(rows, device=dev, generator=g) if case["entropy"] else None
        lse, entropy = [], []
        wide = st["w"].float()
        for x in torch.split(st["x"].float(), max(1, (1 << 27) // vocab)):
            z = x @ wide.T
            lse.append(torch.logsumexp(z, 1))
            entropy.append(lse[-1] - (torch.exp(z - lse[-1][:, None]) * z).sum(1))
        st["lse"], st["entropy"] = torch.cat(lse), torch.cat(entropy)
        st["gx"], st["gw"] = torch.empty_like(st["x"]), torch.empty_like(st["w"])


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    st = {"case": case}
    if case["op"] in ("rotate", "rotate_grad"):
        _prepare_rotate(case, st, g, dev)
    elif case["op"] == "window":
        _prepare_window(case, st, g, dev, torch.Generator().manual_seed(seed))
    else:
        _prepare_score(case, st, g, dev)
    return st


# -------------------------------------------------------------------------- plain forms
def _turn(st):
    """(cos, sin) of every token and pair, [T, 1, rot / 2]: the product wraps at a whole turn."""
    turn = (st["pos"].long()[:, None] * st["freq"]).double() * (2 * math.pi / 2.0 ** 64)
    m = _length(st["case"])
    return (torch.cos(turn) * m).float()[:, None], (torch.sin(turn) * m).float()[:, None]


def _pairs(case, x):
    """The two members of each rotated pair, and the rest of the head."""
    r = case["rot"]
    a, b = (x[..., :r:2], x[..., 1:r:2]) if case["interleaved"] else (x[..., : r // 2], x[..., r // 2:r])
    return a, b, x[..., r:]


def _joined(case, a, b, rest):
    x = torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([x, rest], -1)


def _plain_rotate(st):
    c = st["case"]
    cos, sin = _turn(st)
    for x, w, out in ((st["q"], st["wq"], st["q_out"]), (st["k"], st["wk"], st["k_out"])):
        x = x.float()
        if w is not None:
            x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        a, b, rest = _pairs(c, x)
        out.copy_(_joined(c, a * cos - b * sin, a * sin + b * cos, rest))
    return {"q": st["q_out"], "k": st["k_out"]}


def _plain_rotate_grad(st):
    c = st["case"]
    cos, sin = _turn(st)
    got = {}
    for n, x, w, gy, out in (("q", st["q"], st["wq"], st["gq"], st["q_out"]), ("k", st["k"], st["wk"], st["gk"], st["k_out"])):
        a, b, rest = _pairs(c, gy.float())
        g = _joined(c, a * cos + b * sin, b * cos - a * sin, rest)
        if w is not None:
            x = x.float()
            r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)
            got["w" + n] = (g * x * r).sum((0, 1), dtype=torch.float64).float()
            g = g * w.float()
            g = r * (g - x * (r * r * (g * x).mean(-1, keepdim=True)))
        out.copy_(g)
        got[n] = out
    return got


def _plain_window(st):
    c = st["case"]
    kv, dim, page, q, window, sink = c["kv_heads"], c["dim"], c["page"], c["queries"], c["window"], c["sink"]
    group, dev = c["heads"] // kv, st["q"].device
    start, lens = st["start"].long(), st["lens"].long()
    batch, count = lens.shape[0], start[1:] - start[:-1]
    # the slots that some token of a sequence may see: its first ones, and from the window of its first token on
    first, last = min(sink, c["len"]), min(window + q - 1, c["len"])
    tail = lens[:, None] - last + torch.arange(last, device=dev)
    slot = torch.cat([torch.arange(first, device=dev).expand(batch, first), tail], 1)
    real = slot < lens[:, None]
    real[:, first:] &= (tail >= first) & (tail >= 0)
    slot = torch.where(real, slot, 0)
    at = st["table"].long().gather(1, slot // page)
    gran = st["cache"].view(st["cache"].shape[0], kv, page // 16, 16 * (dim + 8))
    parts = [x.unflatten(-1, (16, -1)) for x in torch.split(gran, [8 * dim, 8 * dim, 64, 64], -1)]
    held = [x[at, :, slot % page // 16, slot % 16] for x in parts]  # [batch, slots, kv heads, bytes of a token]

    def value(codes, grid):
        so = grid.contiguous().view(torch.bfloat16).float()
        x = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() * so[..., :1] + so[..., 1:]
        return x.transpose(1, 2)  # [batch, kv heads, slots, dim]

    k, v = value(held[0], held[2]), value(held[1], held[3])
    i = torch.arange(q, device=dev)
    token = i < count[:, None]
    x = st["q"].float()[torch.where(token, start[:-1, None] + i, 0)]
    x = x.view(batch, q, kv, group, dim).permute(0, 2, 1, 3, 4).reshape(batch, kv, q * group, dim)
    s = torch.matmul(x, k.transpose(2, 3)) / math.sqrt(dim)
    # query i of n sees the slots below its own end, from its window's start on or among the first
    end = lens[:, None] - (count[:, None] - 1 - i)
    seen = real[:, None] & (slot[:, None] < end[:, :, None]) & ((slot[:, None] >= end[:, :, None] - window) | (slot[:, None] < sink))
    seen = seen.repeat_interleave(group, 1)[:, None]
    s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.where(seen, torch.exp(s - torch.where(m > -math.inf, m, 0.0)), 0.0)
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(torch.where(z > 0, p / z, 0.0), torch.where(real[:, None, :, None], v, 0.0))

    def packed(x):
        return x.view(batch, kv, q, group, -1).permute(0, 2, 1, 3, 4).reshape(batch, q, kv * group, -1)[token]

    st["out"].copy_(packed(o))
    st["lse"].copy_(packed(m + torch.log(z))[..., 0])
    return {"out": st["out"], "lse": st["lse"]}


def _plain_score(st):
    z = torch.matmul(st["x"].float(), st["w"].float().T)
    m = z.amax(1, keepdim=True)
    z -= m
    y = st["target"]
    target = z.gather(1, y.clamp(min=0)[:, None])[:, 0]
    e = torch.exp(z)
    total = e.sum(1)
    log_z = torch.log(total)
    entropy = log_z - (e * z).sum(1) / total
    return {"logp": torch.where(y >= 0, target - log_z, 0.0), "entropy": entropy, "lse": m[:, 0] + log_z}


def _plain_grad(st):
    x, w, y = st["x"].float(), st["w"].float(), st["target"]
    lp = torch.matmul(x, w.T) - st["lse"][:, None]
    p = torch.exp(lp)
    g = torch.where(y >= 0, st["g_logp"], 0.0)
    if st["g_entropy"] is not None:
        d = -p * (g[:, None] + st["g_entropy"][:, None] * (lp + st["entropy"][:, None]))
    else:
        d = -p * g[:, None]
    d.scatter_add_(1, y.clamp(min=0)[:, None], g[:, None])
    del p, lp
    st["gx"].copy_(torch.matmul(d, w))
    st["gw"].copy_(torch.matmul(d.T, x))
    return {"gx": st["gx"], "gw": st["gw"]}


# ------------------------------------------------------------------- the framework's calls
def _kept(st, name, make):
    if name not in st:
        st[name] = make()
    return st[name]


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def _own_rotate(kq, st):
    c = st["case"]
    kq.kq_qk_rotate(st["q"], st["k"], st["q_out"], st["k_out"], st["freq"], pos=st["pos"], interleaved=c["interleaved"],
                    scale=_length(c), q_weight=st["wq"], k_weight=st["wk"], eps=EPS)
    return {"q": st["q_out"], "k": st["k_out"]}


def _own_rotate_grad(kq, st):
    c = st["case"]
    sums = {}
    if c["norm"]:
        sums = {n: _kept(st, "sum_" + n, lambda: torch.empty(c["dim"], device="cuda")) for n in ("wq", "wk")}
    ws = _kept(st, "ws", lambda: _bytes(kq.kq_qk_rotate_grad_workspace(st["q"], st["k"])))
    kq.kq_qk_rotate_grad(st["q"], st["k"], st["gq"], st["gk"], st["q_out"], st["k_out"], st["freq"], pos=st["pos"],
                         interleaved=c["interleaved"], scale=_length(c), q_weight=st["wq"], k_weight=st["wk"], eps=EPS,
                         gq_weight=sums.get("wq"), gk_weight=sums.get("wk"), ws=ws)
    return {"q": st["q_out"], "k": st["k_out"], **sums}


def _own_window(kq, st):
    c = st["case"]
    ws = _kept(st, "ws", lambda: _bytes(kq.kq_kv_attend_workspace(st["q"], st["cache"], st["table"])))
    kq.kq_kv_attend_window(st["q"], st["start"], st["lens"], st["cache"], st["table"], st["out"], ws,
                           scale=1 / math.sqrt(c["dim"]), window=c["window"], sink=c["sink"], lse=st["lse"])
    return {"out": st["out"], "lse": st["lse"]}


def _own_score(kq, st):
    got = _kept(st, "results", lambda: {n: torch.empty(st["case"]["rows"], device="cuda") for n in ("logp", "entropy", "lse")})
    ws = _kept(st, "ws", lambda: _bytes(kq.kq_linear_logprobs_workspace(st["x"], st["w"])))
    kq.kq_linear_logprobs(st["x"], st["w"], st["target"], got["logp"], ws, entropy=got["entropy"], lse=got["lse"])
    return got


def _own_grad(kq, st):
    ws = _kept(st, "ws", lambda: _bytes(kq.kq_linear_logprobs_grad_workspace(st["x"], st["w"])))
    kq.kq_linear_logprobs_grad(st["x"], st["w"], st["target"], st["lse"], st["g_logp"], ws, gx=st["gx"], gw=st["gw"],
                               entropy=st["entropy"], g_entropy=st["g_entropy"])
    return {"gx": st["gx"], "gw": st["gw"]}


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2607_07964_gb300 import kronq as kq
        return {"rotate": _own_rotate, "rotate_grad": _own_rotate_grad, "window": _own_window, "score": _own_score,
                "grad": _own_grad}[op](kq, state)
    return {"rotate": _plain_rotate, "rotate_grad": _plain_rotate_grad, "window": _plain_window, "score": _plain_score,
            "grad": _plain_grad}[op](state)


# ---------------------------------------------------------------------------------- work
def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    op = case["op"]
    if op in ("score", "grad"):
        rows, vocab, hidden = case["rows"], case["vocab"], case["hidden"]
        size, product = 2 * hidden * (rows + vocab), 2 * rows * vocab * hidden
        return {"bytes": size + 20 * rows, "flops": product} if op == "score" else {"bytes": 2 * size + 24 * rows, "flops": 3 * product}
    size, dim = 2 if case["dtype"] == "bf16" else 4, case["dim"]
    if op in ("rotate", "rotate_grad"):
        n = case["tokens"] * (case["heads"] + case["kv_heads"]) * dim
        return {"bytes": (3 if op == "rotate_grad" else 2) * n * size + 4 * case["tokens"], "flops": (14 if op == "rotate_grad" else 7) * n}
    # lengths are spread between a quarter of the longest and it; queries between one and their most
    batch, most = case["batch"], case["window"] + case["sink"]
    each = [max(1, int(case["len"] * (0.25 + 0.75 * (0.618034 * i % 1)))) for i in range(1, batch)] + [case["len"]]
    slots = case["kv_heads"] * sum(min(n, most) for n in each)
    rows = batch * (case["queries"] + 1) / 2 * case["heads"]
    return {"bytes": slots * (dim + 8) + rows * (2 * dim * size + 4), "flops": 4 * slots * rows / batch / case["kv_heads"] * dim}


# ------------------------------------------------------------------- 64 bits, written apart
def _exact_rotate(case, st):
    """Rotations as products of complex numbers."""
    n = case["rot"]
    angle = st["pos"].double()[:, None] * torch.tensor(_theta(case), dtype=torch.float64, device=st["pos"].device)
    unit = torch.polar(torch.full_like(angle, _length(case)), angle)[:, None]
    back = case["op"] == "rotate_grad"
    got = {}
    for name, x, w, gy in (("q", st["q"], st["wq"], st.get("gq")), ("k", st["k"], st["wk"], st.get("gk"))):
        x = x.double()
        norm = (x.pow(2).sum(-1, keepdim=True) / case["dim"] + EPS).rsqrt() if w is not None else None
        y = gy.double().clone() if back else x.clone() if w is None else x * norm * w.double()
        re, im = (slice(0, n, 2), slice(1, n, 2)) if case["interleaved"] else (slice(0, n // 2), slice(n // 2, n))
        z = torch.complex(y[..., re], y[..., im]) * (unit.conj() if back else unit)
        y[..., re], y[..., im] = z.real, z.imag
        if back and w is not None:
            hat = x * norm
            got["w" + name] = torch.einsum("thd,thd->d", y, hat)
            y = y * w.double()
            y = norm * (y - hat * (y * hat).sum(-1, keepdim=True) / case["dim"])
        got[name] = y
    return got


def _exact_window(case, st):
    """Sequence by sequence, head by head, on the slots themselves."""
    kv, dim, page = case["kv_heads"], case["dim"], case["page"]
    group, dev = case["heads"] // kv, st["q"].device
    out = torch.zeros(st["q"].shape[0], case["heads"], dim, dtype=torch.float64, device=dev)
    lse = torch.full((st["q"].shape[0], case["heads"]), -math.inf, dtype=torch.float64, device=dev)
    start, lens = st["start"].tolist(), st["lens"].tolist()
    d = torch.arange(dim, device=dev)
    for b, n in enumerate(lens):
        count = start[b + 1] - start[b]
        low = max(0, n - count + 1 - case["window"])
        t = torch.tensor([j for j in range(min(case["sink"], n))] + list(range(max(low, min(case["sink"], n)), n)), dtype=torch.long, device=dev)
        if not n:
            continue
        held = st["cache"][st["table"][b].long()[t // page]]  # [slots, heads, bytes of a page and head]
        base = (t % page // 16) * 16 * (dim + 8)

        def values(which):
            at = base[:, None] + which * 8 * dim + (t % 16)[:, None] * (dim // 2) + d // 2
            byte = held.gather(2, at[:, None].expand(-1, kv, -1)).int()
            code = torch.where(d % 2 == 0, byte % 16, byte // 16).double()
            at = base[:, None] + 16 * dim + which * 64 + (t % 16)[:, None] * 4 + torch.arange(4, device=dev)
            w = held.gather(2, at[:, None].expand(-1, kv, -1)).int()
            scale, offset = (((w[..., i + 1] * 256 + w[..., i]) << 16).view(torch.float32).double() for i in (0, 2))
            return code * scale[..., None] + offset[..., None]

        k, v = values(0), values(1)
        for i in range(count):
            m = n - (count - 1 - i)
            see = (t < m) & ((t >= m - case["window"]) | (t < case["sink"]))
            if not see.any():
                continue
            x = st["q"][start[b] + i].double().view(kv, group, dim)
            s = torch.einsum("hgd,shd->hgs", x, k[see]) / math.sqrt(dim)
            z = torch.logsumexp(s, -1)
            lse[start[b] + i] = z.flatten()
            out[start[b] + i] = torch.einsum("hgs,shd->hgd", torch.exp(s - z[..., None]), v[see]).reshape(-1, dim)
    return {"out": out, "lse": lse}


def exact(case, seed):
    if case["op"] in ("score", "grad") and work(case)["flops"] > 1e13:
        return None
    st = prepare(case, seed)
    if case["op"] in ("rotate", "rotate_grad"):
        return _exact_rotate(case, st)
    if case["op"] == "window":
        return _exact_window(case, st)
    x, w, y = st["x"].double(), st["w"].double(), st["target"]
    scored = (y >= 0).nonzero()[:, 0]
    if case["op"] == "score":
        logp, entropy, lse = (torch.zeros(x.shape[0], dtype=torch.float64, device=x.device) for _ in range(3))
        for i in torch.split(torch.arange(x.shape[0], device=x.device), 1024):
            lp = torch.log_softmax(x[i] @ w.T, 1)
            lse[i] = (x[i] * w[0]).sum(1) - lp[:, 0]
            entropy[i] = -(lp.exp() * lp).sum(1)
            logp[i] = lp.gather(1, y[i].clamp(min=0)[:, None])[:, 0]
        return {"logp": torch.where(y >= 0, logp, 0.0), "entropy": entropy, "lse": lse}
    gx, gw = torch.zeros_like(x), torch.zeros_like(w)
    for i in torch.split(torch.arange(x.shape[0], device=x.device), 1024):
        lp = x[i] @ w.T - st["lse"][i].double()[:, None]
        p = lp.exp()
        if st["g_entropy"] is not None:
            d = -st["g_entropy"][i].double()[:, None] * p * (lp + st["entropy"][i].double()[:, None])
        else:
            d = torch.zeros_like(p)
        g = torch.where(y[i] >= 0, st["g_logp"][i], 0.0).double()
        d -= g[:, None] * p
        d[torch.arange(len(i), device=x.device), y[i].clamp(min=0)] += g
        gx[i] = d @ w
        gw += d.T @ x[i]
    return {"gx": gx, "gw": gw}
