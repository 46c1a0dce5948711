"""The 4-bit key/value cache in numpy: quantizer and layout with the float32 operations that define
the codes, attention and eviction in 64 bits. Test infrastructure only."""
import numpy as np

GRANULE = 16


def quantize(x):
    """codes uint8 [..., D], (scale, offset) float32 [..., 2] of rows x float32 [..., D]."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        lo, hi = x.min(-1), x.max(-1)
        b = np.ascontiguousarray(lo).view(np.uint32)
        ob = (b + np.where(b >> 31, 0xFFFF, 0).astype(np.uint32)) & np.uint32(0xFFFF0000)
        off = ob.view(np.float32)
        s = np.ascontiguousarray((hi - off) / np.float32(15))
        s = ((s.view(np.uint32) + np.uint32(0xFFFF)) & np.uint32(0xFFFF0000)).view(np.float32)
        ok = np.isfinite(x).all(-1) & np.isfinite(off) & np.isfinite(s)
        c = np.clip(np.rint((x - off[..., None]) / s[..., None]), 0, 15)
        c = np.where((ok & (s > 0))[..., None], c, 0).astype(np.uint8)
        nan = np.float32(np.nan)
        return c, np.stack([np.where(ok, s, nan), np.where(ok, off, nan)], -1)


def param_bytes(so):
    u = np.ascontiguousarray(so.astype(np.float32)).view(np.uint32) >> 16
    u = np.where(np.isnan(so), 0x7FC0, u).astype(np.uint16)
    return u.view(np.uint8).reshape(*so.shape[:-1], 4)


class Cache:
    """A pool in numpy, data [pages, heads, page * (dim + 8)], with table [batch, pages of a sequence]."""

    def __init__(self, data, table, page, dim):
        self.data, self.table, self.page, self.dim = data, table, page, dim

    def _at(self, b, h, slot):
        base = self.data[self.table[b, slot // self.page], h]
        g = slot % self.page // GRANULE * GRANULE * (self.dim + 8)
        return base[g:g + GRANULE * (self.dim + 8)], slot % GRANULE

    def views(self, b, h, slot, which):
        g, t = self._at(b, h, slot)
        half = self.dim // 2
        code = which * GRANULE * half + t * half
        par = GRANULE * self.dim + which * GRANULE * 4 + t * 4
        return g[code:code + half], g[par:par + 4]

    def put(self, b, h, slot, which, row):
        c, so = (x[0] for x in quantize(row[None]))
        code, par = self.views(b, h, slot, which)
        code[:] = c[::2] | (c[1::2] << 4)
        par[:] = param_bytes(so)

    def rows(self, b, h, n, which):
        """values, and the magnitude 15 |scale| + |offset| of each row, in 64 bits"""
        out, mag = np.zeros((n, self.dim)), np.zeros(n)
        for j in range(n):
            code, par = self.views(b, h, j, which)
            so = (np.ascontiguousarray(par).view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
            out[j, ::2], out[j, 1::2] = code & 15, code >> 4
            out[j] = out[j] * so[0] + so[1]
            mag[j] = 15 * abs(so[0]) + abs(so[1])
        return out, mag

    def move(self, b, h, src, dst):
        for which in range(2):
            for d, s in zip(self.views(b, h, dst, which), self.views(b, h, src, which)):
                d[:] = s


def attend(cache, q, start, lens, kv_heads, scale):
    """out, lse, weight [batch, heads, slots], and the error scales: score [T, Hq] (the largest score's terms in
    absolute value) and value [T, Hq] (sum of weight times magnitude of the values)."""
    T, Hq, D = q.shape
    G = Hq // kv_heads
    S = cache.table.shape[1] * cache.page
    out, lse = np.zeros((T, Hq, D)), np.full((T, Hq), -np.inf)
    weight, werr = np.zeros((len(lens), kv_heads, S)), np.zeros((len(lens), kv_heads, S))
    es, ev = np.zeros((T, Hq)), np.zeros((T, Hq))
    for b, n in enumerate(lens):
        for h in range(kv_heads):
            k, mk = cache.rows(b, h, n, 0)
            v, mv = cache.rows(b, h, n, 1)
            for i in range(start[b], start[b + 1]):
                m = n - (start[b + 1] - 1 - i)
                if m <= 0:
                    continue
                for g in range(G):
                    x = q[i, h * G + g].astype(np.float64)
                    with np.errstate(all="ignore"):
                        s = scale * (k[:m] @ x)
                        top = s.max()
                        e = np.exp(s - top)
                        p = e / e.sum()
                        out[i, h * G + g] = p @ v[:m]
                        lse[i, h * G + g] = top + np.log(e.sum())
                        es[i, h * G + g] = abs(scale) * np.abs(x).sum() * mk[:m].max()
                        ev[i, h * G + g] = p @ mv[:m]
                    weight[b, h, :m] += p
                    werr[b, h, :m] += p * es[i, h * G + g]
    return out, lse, weight, es, ev, werr


def evict(acc, pos, n, seen, budget, recent, sink):
    """The slot that each kept place takes its content from, for one sequence and head."""
    if n <= budget:
        return list(range(n))
    safe = [pos[j] >= seen - recent or pos[j] < sink for j in range(n)]

    def order(j):
        if safe[j]:
            return (0, 0.0, j)
        return (2, 0.0, j) if np.isnan(acc[j]) else (1, -float(acc[j]), j)

    keep = set(sorted(range(n), key=order)[:budget])
    tail = iter(sorted(j for j in keep if j >= budget))
    return [j if j in keep else next(tail) for j in range(budget)]
