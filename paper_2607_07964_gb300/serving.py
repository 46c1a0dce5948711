"""Decoding with quantized layers over a 4-bit key/value cache, and scoring what was decoded.

QuantizedLinear applies a layer that LayerPipeline quantized (kq_pack_codes, kq_infer);
KvCache owns a pool of pages and strings together kq_kv_append, kq_kv_attend, kq_kv_evict and
kq_kv_read for a batch of sequences; AttentionBlock is one attention sublayer over both, without the
norm before it and the rotation of queries and keys, which a model puts around and between. Products,
cache, attention and scoring run in libkronq's kernels, on the current stream, without waiting for the
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

    def attend(self, q, start, scale: float | None = None, lse=None):
        """Attention of q [T, q_heads, dim] of the tokens appended last over their sequences."""
        self._capturing()
        need = kq.kq_kv_attend_workspace(q, self.data, self.table, self.acc)
        if self._ws is None or self._ws.numel() < need:
            if self._fixed:
                self._held.append(self._ws)
            elif self._ws is not None:   # may have been made on another stream than the one that uses it last
                self._ws.record_stream(torch.cuda.current_stream())
            self._ws = torch.empty(need, dtype=torch.uint8, device=q.device)
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        kq.kq_kv_attend(q, start, self.lens, self.data, self.table, out, self._ws,
                        1 / math.sqrt(self.dim) if scale is None else scale, lse=lse, acc=self.acc, info=self.info)
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


class AttentionBlock:
    """x + W_o attention(W_q x, W_k x, W_v x) with quantized projections, tokens of several sequences packed (start and
    most as KvCache.append takes them). Queries and keys are not rotated."""

    def __init__(self, proj: dict, heads: int, cache: KvCache):
        self.proj, self.heads, self.cache = proj, heads, cache

    def __call__(self, x, start, most):
        c, T = self.cache, x.shape[0]
        q, k, v = (self.proj[n](x) for n in ("q", "k", "v"))
        c.append(k.view(T, c.kv_heads, c.dim), v.view(T, c.kv_heads, c.dim), start, most)
        a = c.attend(q.view(T, self.heads, c.dim), start)
        return x + self.proj["o"](a.view(T, -1))


def score(logits, target, top: int = 0):
    """(logp, entropy, top_id, top_logp) of the target tokens under logits [T, V]."""
    T, dev = logits.shape[0], logits.device
    logp, entropy = torch.empty(T, device=dev), torch.empty(T, device=dev)
    ids = torch.empty(T, top, dtype=torch.int32, device=dev) if top else None
    tops = torch.empty(T, top, device=dev) if top else None
    kq.kq_token_logprobs(logits, target, logp, entropy=entropy, top_id=ids, top_logp=tops)
    return logp, entropy, ids, tops


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
            budget: int = 32, bits: int = 4, seed: int = 0):
    """Prompts of different lengths, then `steps` greedily decoded tokens of each under a cache budget. Returns
    the decoded tokens and their log probabilities [steps, batch], and the block."""
    d, batch = heads * dim, len(prompts)
    proj = {n: _quantized(n, d if n in "qo" else kv_heads * dim, d, bits, seed + i) for i, n in enumerate("qkvo")}
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
