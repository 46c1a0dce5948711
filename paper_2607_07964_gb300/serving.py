"""Decoding with quantized layers over a 4-bit key/value cache, and scoring what was decoded.

QuantizedLinear applies a layer that LayerPipeline quantized (kq_pack_codes, kq_infer);
KvCache owns a pool of pages and strings together kq_kv_append, kq_kv_attend, kq_kv_attend_window,
kq_kv_evict and kq_kv_read for a batch of sequences; Rotation holds the positions' frequencies and the
norms of queries and keys (kq_qk_rotate); AttentionBlock is one attention sublayer over them, without the
norm before it, which a model puts around it; score takes logits, score_hidden the hidden states and the
head that they would come from, score_hidden_grad the gradients. Products, cache, attention and
scoring run in libkronq's kernels, on the current stream, without waiting for the
device (`KvCache.append` says when it has to); `KvCache.check` reads the device error word.

`python -m paper_2607_07964_gb300.serving` quantizes the projections of a small random model,
feeds prompts of different lengths, decodes greedily with eviction, and prints the log
probabilities of the decoded tokens.
"""
from __future__ import annotations

import math

import torch

from . import kronq as kq


class QuantizedLinear:
    """y = W^ x for up to 8 tokens a call, from a finished LayerPipeline."""

    def __init__(self, pipe, sign_u, sign_v, bits: int, group: int):
        self.d_out, self.d_in = pipe.codes.shape
        self.bits, self.group = bits, group
        self.packed = torch.empty(kq.kq_packed_codes_bytes(self.d_out, self.d_in, bits) // 4, dtype=torch.int32,
                                  device=pipe.codes.device)
        kq.kq_pack_codes(pipe.codes, bits, self.packed)
        self.scale, self.zero = pipe.scale.clone(), pipe.zero.clone()
        self.s_x, self.s_g = pipe.s_x.clone(), pipe.s_g.clone()
        self.sign_u, self.sign_v = sign_u, sign_v
        self.ws = torch.empty(kq.kq_infer_workspace(8, self.d_in, self.d_out), dtype=torch.uint8, device=pipe.codes.device)

    def __call__(self, x):
        y = torch.empty(x.shape[0], self.d_out, device=x.device)
        for i in range(0, x.shape[0], 8):
            kq.kq_infer(self.packed, self.scale, self.zero, self.d_out, self.d_in, self.bits, self.group, self.s_x, self.s_g,
                        self.sign_u, self.sign_v, x[i:i + 8], y[i:i + 8], self.ws)
        return y


def _check_window(cache, window: int, sink: int) -> None:
    if cache.budget is not None:
        raise ValueError("a cache that evicts does not hold its slots in the order of positions, so it has no window")
    if window < 1 or sink < 0:
        raise ValueError(f"window must be at least 1 and sink at least 0, got {window} and {sink}")


class KvCache:
    """The 4-bit cache of `batch` sequences with up to `slots` cached tokens each. With a budget, append
    first cuts the sequences back to `budget` slots when the new tokens would not fit: the last `recent` and
    first `sink` positions stay, and those that drew the most attention weight since they were
    cached, each head on its own.

    Its calls can be captured in CUDA graphs and replayed on the lengths as they then are. The host does not see
    replays: once an append has been captured, the others read the lengths from the device first, and replays past the
    last slot are up to the caller (a captured `evict` keeps away from it; tokens without a slot are reported by `check`)."""

    def __init__(self, batch: int, kv_heads: int, dim: int, slots: int, page: int = 64, budget: int | None = None,
                 recent: int = 0, sink: int = 0, device: str = "cuda"):
        if budget is not None and not 0 < budget <= slots:
            raise ValueError("budget must be between 1 and slots")
        per = -(-slots // page)
        i32 = dict(dtype=torch.int32, device=device)
        self.kv_heads, self.dim, self.slots = kv_heads, dim, slots
        self.budget, self.recent, self.sink = budget, recent, sink
        self.data = torch.zeros(batch * per, kv_heads, kq.kq_kv_cache_bytes(page, dim), dtype=torch.uint8, device=device)
        self.table = torch.arange(batch * per, **i32).view(batch, per)
        self.lens, self._lens = torch.zeros(batch, **i32), torch.zeros(batch, **i32)
        self.seen, self._seen = torch.zeros(batch, **i32), torch.zeros(batch, **i32)
        self.info = torch.zeros(1, **i32)
        self.acc = self.pos = self._evict_ws = None
        if budget is not None:
            self.acc = torch.zeros(batch, kv_heads, slots, device=device)
            self.pos = torch.zeros(batch, kv_heads, slots, **i32)
            self._evict_ws = torch.empty(kq.kq_kv_evict_workspace(self.acc, budget), dtype=torch.uint8, device=device)
        self._ws, self._held = None, []   # workspaces that a graph may write to stay
        # what the host knows of the lengths: a sequence holds at most its entry and what all may have got since
        self._each, self._peak, self._all = [0] * batch, 0, 0
        self._sure = True   # exactly that
        self._fixed = False     # a graph holds the arrays
        self._replayed = False   # and may have appended since

    @property
    def most(self) -> int:
        """Slots that the longest sequence may hold."""
        return self._peak + self._all

    def _account(self, each) -> None:
        self._each, self._peak, self._all = each, max(each), 0

    def _longest(self, more, cap: int | None = None) -> int:
        """The longest sequence's slots after `more` tokens, a number for all or a list, first cut back to `cap`."""
        def left(n):
            return n if cap is None else min(n, cap)
        if not isinstance(more, list):
            return left(self.most) + more
        return max(left(n + self._all) + m for n, m in zip(self._each, more))

    def _capturing(self) -> bool:
        now = self.lens.is_cuda and torch.cuda.is_current_stream_capturing()
        self._fixed = self._fixed or now
        return now

    def _take(self, seen: bool) -> None:
        """The lengths (and counts) that a call has written become the current ones: they change places, which costs
        nothing, or are copied where a graph holds the arrays."""
        if self._fixed:
            self.lens.copy_(self._lens)
            if seen:
                self.seen.copy_(self._seen)
            return
        self.lens, self._lens = self._lens, self.lens
        if seen:
            self.seen, self._seen = self._seen, self.seen

    def measure(self) -> None:
        """Reads the lengths from the device."""
        self._account(self.lens.tolist())
        self._sure = True

    def append(self, k, v, start, most) -> None:
        """k, v [T, kv_heads, dim] of the sequences' next tokens; start [batch + 1] on the device; most: the
        largest number of tokens that a sequence gets, or a list of the number that each gets. Where the largest
        number leaves open whether the tokens fit, the lengths are read from the device."""
        batch, T = len(self._each), k.shape[0]
        more = list(most) if isinstance(most, (list, tuple)) else most
        sure = isinstance(more, list) or T == batch * more
        if isinstance(more, list) and (len(more) != batch or min(more) < 0 or sum(more) != T):
            raise ValueError(f"most must be a number or {batch} counts that add up to the {T} tokens of k, got {most}")
        capturing = self._capturing()
        if self._replayed and not capturing:
            self.measure()
        self._replayed = self._replayed or capturing
        if self._longest(more) > self.slots:
            if not (self._sure and sure) and not capturing:
                self.measure()
                ends = start.tolist()
                more, sure = [b - a for a, b in zip(ends, ends[1:])], True
            if self._longest(more) > self.slots:
                if self.budget is None or self._longest(more, self.budget) > self.slots:
                    raise ValueError(f"{most} more tokens do not fit {self.slots} slots")
                self.evict()
        kq.kq_kv_append(k, v, start, self.lens, self.data, self.table, lens_out=self._lens, acc=self.acc, pos=self.pos,
                        seen=self.seen, seen_out=self._seen, info=self.info)
        self._take(seen=True)
        self._sure = self._sure and sure
        if isinstance(more, list):
            self._account([n + self._all + m for n, m in zip(self._each, more)])
        else:
            self._all += more

    def attend(self, q, start, scale: float | None = None, lse=None, window: int | None = None, sink: int = 0):
        """Attention of q [T, q_heads, dim] of the tokens appended last over their sequences; with a window, over the last
        `window` positions up to a token's own and the first `sink`, without one over all of them."""
        if window is not None:
            _check_window(self, window, sink)
        self._capturing()
        need = kq.kq_kv_attend_workspace(q, self.data, self.table, self.acc)
        if self._ws is None or self._ws.numel() < need:
            if self._fixed:
                self._held.append(self._ws)
            elif self._ws is not None:   # may have been made on another stream than the one that uses it last
                self._ws.record_stream(torch.cuda.current_stream())
            self._ws = torch.empty(need, dtype=torch.uint8, device=q.device)
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        scale = 1 / math.sqrt(self.dim) if scale is None else scale
        if window is None:
            kq.kq_kv_attend(q, start, self.lens, self.data, self.table, out, self._ws, scale, lse=lse, acc=self.acc, info=self.info)
        else:
            kq.kq_kv_attend_window(q, start, self.lens, self.data, self.table, out, self._ws, scale, window, sink, lse=lse,
                                   info=self.info)
        return out

    def evict(self) -> None:
        """Cuts every sequence with more than `budget` slots back to it."""
        if self.budget is None:
            raise ValueError("a cache without a budget has nothing to cut back to")
        self._capturing()
        kq.kq_kv_evict(self.data, self.table, self.lens, self.acc, self.pos, self.seen, self.dim, self.budget, self.recent,
                       self.sink, self._lens, self.acc, self.pos, self._evict_ws, info=self.info)
        self._take(seen=False)
        self._account([min(n + self._all, self.budget) for n in self._each])

    def read(self, dtype=torch.float32):
        """The cached keys and values, [batch, slots, kv_heads, dim], zeros past each length."""
        self._capturing()
        batch = self.lens.shape[0]
        start = torch.arange(0, (batch + 1) * self.slots, self.slots, dtype=torch.int32, device=self.lens.device)
        k, v = (torch.empty(batch * self.slots, self.kv_heads, self.dim, dtype=dtype, device=self.lens.device) for _ in range(2))
        kq.kq_kv_read(self.data, self.table, start, None, self.lens, k, v, info=self.info)
        return tuple(t.view(batch, self.slots, self.kv_heads, self.dim) for t in (k, v))

    def check(self) -> None:
        status, raw = kq.kq_check(self.info)
        if status != kq.KQ_OK:
            raise kq.KronqError(status, "KvCache", f"device error word {raw}")


def rotation_theta(rot: int, base: float = 10000.0, stretch: float = 1.0, original: int = 8192):
    """Radians that one position turns the pairs of `rot` dimensions by, base^(-2 j / rot), and the scale of queries and keys.
    With stretch > 1, for texts of up to `stretch` times the `original` positions: waves that the original length
    holds less than once are slowed by stretch, those that it holds four times or more are kept, those between in
    proportion, and queries and keys are scaled by 1 + ln(stretch) / 10 each."""
    theta = []
    for j in range(rot // 2):
        t = base ** (-2 * j / rot)
        keep = min(1.0, max(0.0, (original * t / (2 * math.pi) - 1) / 3))
        theta.append(t * (keep + (1 - keep) / stretch))
    return theta, 1.0 + 0.1 * math.log(stretch)


class Rotation:
    """The rotation of queries and keys by their positions, and their norms before it where there are weights: theta and scale as
    rotation_theta gives them."""

    def __init__(self, theta, scale: float = 1.0, interleaved: bool = False, q_weight=None, k_weight=None, eps: float = 1e-6,
                 device: str = "cuda"):
        self.freq = kq.kq_rotation_freq(theta, device)
        self.args = dict(scale=scale, interleaved=interleaved, q_weight=q_weight, k_weight=k_weight, eps=eps)

    def __call__(self, q, k, **positions) -> None:
        """q, k [T, heads, dim] in place; positions: pos [T], or start and first."""
        kq.kq_qk_rotate(q, k, q, k, self.freq, **positions, **self.args)

    def grad(self, q, k, gq, gk, **positions):
        """(gradients of the weights, of queries and of keys, None without weights) for q, k as they were before the rotation; gq, gk,
        the gradients of what it made of them, become those of q and k in place."""
        sums = [None if g is None or self.args[n] is None else torch.empty(gq.shape[2], device=gq.device)
                for n, g in (("q_weight", gq), ("k_weight", gk))]
        ws = torch.empty(kq.kq_qk_rotate_grad_workspace(gq), dtype=torch.uint8, device=gq.device) if any(
            s is not None for s in sums) else None
        kq.kq_qk_rotate_grad(q, k, gq, gk, gq, gk, self.freq, gq_weight=sums[0], gk_weight=sums[1], ws=ws, **positions, **self.args)
        return tuple(sums)


class AttentionBlock:
    """x + W_o attention(W_q x, W_k x, W_v x) with quantized projections, tokens of several sequences packed (start and
    most as KvCache.append takes them). Queries and keys are normed and rotated where a Rotation is given, by the number of
    tokens that their sequence has had; with a window, attention sees the last `window` positions and the first `sink`, without
    one all of them."""

    def __init__(self, proj: dict, heads: int, cache: KvCache, rotation: Rotation | None = None, window: int | None = None,
                 sink: int = 0):
        # here, as a step that fails in its attention has appended its tokens
        if window is not None:
            _check_window(cache, window, sink)
        self.proj, self.heads, self.cache = proj, heads, cache
        self.rotation, self.window, self.sink = rotation, window, sink

    def __call__(self, x, start, most):
        c, T = self.cache, x.shape[0]
        q, k, v = (self.proj[n](x) for n in ("q", "k", "v"))
        q, k, v = q.view(T, self.heads, c.dim), k.view(T, c.kv_heads, c.dim), v.view(T, c.kv_heads, c.dim)
        if self.rotation is not None:
            self.rotation(q, k, start=start, first=c.seen)
        c.append(k, v, start, most)
        a = c.attend(q, start, window=self.window, sink=self.sink)
        return x + self.proj["o"](a.view(T, -1))


def score(logits, target, top: int = 0):
    """(logp, entropy, top_id, top_logp) of the target tokens under logits [T, V]."""
    T, dev = logits.shape[0], logits.device
    logp, entropy = torch.empty(T, device=dev), torch.empty(T, device=dev)
    ids = torch.empty(T, top, dtype=torch.int32, device=dev) if top else None
    tops = torch.empty(T, top, device=dev) if top else None
    kq.kq_token_logprobs(logits, target, logp, entropy=entropy, top_id=ids, top_logp=tops)
    return logp, entropy, ids, tops


def score_hidden(x, head, target, info=None):
    """(logp, entropy, lse) of the target tokens under the logits x head^T of hidden states x [T, d] and a head [V, d] (bf16), as
    score gives them for logits, which are not made here."""
    T, dev = x.shape[0], x.device
    logp, entropy, lse = (torch.empty(T, device=dev) for _ in range(3))
    ws = torch.empty(kq.kq_linear_logprobs_workspace(x, head), dtype=torch.uint8, device=dev)
    kq.kq_linear_logprobs(x, head, target, logp, ws, entropy=entropy, lse=lse, info=info)
    return logp, entropy, lse


def score_hidden_grad(x, head, target, lse, g_logp, entropy=None, g_entropy=None, of_head: bool = True, info=None):
    """(gx, gradient of the head or None) of sum(g_logp * logp + g_entropy * entropy), from score_hidden's lse and entropy: with
    g_logp = -1 / T what calibration starts its backward pass from."""
    gx, gw = torch.empty_like(x), torch.empty_like(head) if of_head else None
    ws = torch.empty(kq.kq_linear_logprobs_grad_workspace(x, head), dtype=torch.uint8, device=x.device)
    kq.kq_linear_logprobs_grad(x, head, target, lse, g_logp, ws, gx=gx, gw=gw, entropy=entropy if g_entropy is not None else None,
                               g_entropy=g_entropy, info=info)
    return gx, gw


def _quantized(name: str, d_out: int, d_in: int, bits: int, seed: int) -> QuantizedLinear:
    """A random layer quantized on random calibration data, d_out and d_in with a Hadamard construction."""
    from .pipeline import LayerPipeline
    g = torch.Generator("cuda").manual_seed(seed)
    X, G = (torch.randn(1024, d, device="cuda", generator=g).bfloat16() for d in (d_in, d_out))
    W = torch.randn(d_out, d_in, device="cuda", generator=g) / math.sqrt(d_in)
    su, sv = ((torch.randint(0, 2, (d,), device="cuda", generator=g) * 2 - 1).to(torch.int8) for d in (d_out, d_in))
    pipe = LayerPipeline(d_out, d_in, bits, 128, 128, 0.01, device="cuda")
    pipe.run(X, G, W, su, sv)
    pipe.check()
    return QuantizedLinear(pipe, su, sv, bits, 128)


def example(steps: int = 24, prompts=(40, 7, 23), vocab: int = 1000, heads: int = 4, kv_heads: int = 2, dim: int = 128,
            budget: int | None = 32, bits: int = 4, seed: int = 0, window: int | None = None):
    """Prompts of different lengths, then `steps` greedily decoded tokens of each: under a cache budget, or (budget None) with rotated
    queries and keys and a window. Returns the decoded tokens and their log probabilities [steps, batch], and the block."""
    d, batch = heads * dim, len(prompts)
    proj = {n: _quantized(n, d if n in "qo" else kv_heads * dim, d, bits, seed + i) for i, n in enumerate("qkvo")}
    if budget is None:
        cache = KvCache(batch, kv_heads, dim, max(prompts) + steps)
        one = torch.ones(dim, device="cuda")
        theta, scale = rotation_theta(dim)
        block = AttentionBlock(proj, heads, cache, Rotation(theta, scale, q_weight=one, k_weight=one), window, sink=2)
    else:
        cache = KvCache(batch, kv_heads, dim, max(max(prompts), budget) + 8, budget=budget, recent=budget // 4, sink=2)
        block = AttentionBlock(proj, heads, cache)
    g = torch.Generator("cuda").manual_seed(seed)
    embed, head = (torch.randn(vocab, d, device="cuda", generator=g) for _ in range(2))
    tokens = torch.randint(0, vocab, (sum(prompts),), device="cuda", generator=g)
    ends = torch.tensor((0,) + tuple(prompts), device="cuda").cumsum(0).to(torch.int32)
    x = block(embed[tokens], ends, prompts)[(ends[1:] - 1).long()]
    one = torch.arange(batch + 1, dtype=torch.int32, device="cuda")
    ids, logps = [], []
    for _ in range(steps):
        logits = x @ head.T / math.sqrt(d)
        logp, _, top_id, _ = score(logits, tokens.new_zeros(batch), top=1)
        tokens = top_id[:, 0].long()
        logp, _, _, _ = score(logits, tokens)
        ids.append(tokens)
        logps.append(logp)
        x = block(embed[tokens], one, 1)
    cache.check()
    return torch.stack(ids), torch.stack(logps), block


if __name__ == "__main__":
    ids, logps, block = example()
    c = block.cache
    print(f"decoded {ids.shape[0]} tokens of {ids.shape[1]} sequences, mean log probability {logps.mean().item():.3f}")
    print(f"cache: {c.lens.tolist()} slots of {c.seen.tolist()} tokens seen, {c.data.numel()} bytes "
          f"({c.data.numel() / (2 * c.table.numel() * 64 * c.kv_heads * c.dim) * 8:.2f} bits a value)")
