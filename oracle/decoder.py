"""The decoder operators (root-mean-square norm, cache in 4 bits) from their definitions, in numpy's 64-bit integers.

Test infrastructure, like the rest of this folder: nothing here is shared with the CUDA library.  Scales are (mult, shift), numbers or
arrays with an entry per channel.
"""
import math

import numpy as np

_i = np.int64


def rq(a, mult, shift):
    """floor((a mult + 2^(shift-1)) / 2^shift); |a mult| < 2^62."""
    m, s = _i(mult) if np.isscalar(mult) else np.asarray(mult, _i), _i(shift) if np.isscalar(shift) else np.asarray(shift, _i)
    return (np.asarray(a, _i) * m + (_i(1) << (s - 1))) >> s


def shiftexp(n, I0, N):
    """Algorithm 1's ShiftExp(-n), n >= 0."""
    n = np.asarray(n, _i)
    t = n + (n + 1) // 2 - (n + 15) // 16        # -(I + (I >> 1) - (I >> 4)) at I = -n
    q, r = t // I0, t % I0
    mant = I0 - (r + 1) // 2
    return np.where(q <= N, mant << np.clip(N - q, 0, 62), mant >> np.clip(q - N, 0, 62))


def rmsnorm(x, gamma, M_ln, x_scale=None, res=None, res_scale=None, stream_i32=False, dynamic=False):
    """(out, row_max or None, sum or None)."""
    if res is None:
        h = np.clip(np.asarray(x, _i), -(1 << 20), 1 << 20)
    else:
        lo, hi = (-(1 << 20), 1 << 20) if stream_i32 else (-128, 127)
        h = np.clip(rq(x, *x_scale) + rq(res, *res_scale), lo, hi)
    out, tops = np.zeros(h.shape, _i), np.zeros(h.shape[0], _i)
    for r, row in enumerate(h):
        sd = math.isqrt(int((row * row).sum()))
        e = sd.bit_length()
        y = (row * _i((1 << (M_ln + e)) // sd) + (_i(1) << (e - 1))) >> e if sd else 0 * row
        z = rq(y, *gamma)
        tops[r] = A = int(np.abs(z).max())
        k = 23 + A.bit_length()
        out[r] = ((z * _i((127 << k) // A) + (_i(1) << (k - 1))) >> k if A else 0) if dynamic else np.clip(z, -128, 127)
    return out, (tops if dynamic else None), (h if res is not None else None)


class Cache:
    """Codes and steps of a pool as whole numbers: kc, vc [pages, heads, page, d], ks [.., d/32], vs [..]."""

    def __init__(self, pages, heads, d, page):
        self.d, self.page = d, page
        self.kc, self.vc = np.zeros((pages, heads, page, d), _i), np.zeros((pages, heads, page, d), _i)
        self.ks, self.vs = np.zeros((pages, heads, page, d // 32), _i), np.zeros((pages, heads, page), _i)

    @classmethod
    def of_bytes(cls, pool, d, page):
        """What the bytes of a pool [pages, heads, bytes] stand for."""
        c = cls(pool.shape[0], pool.shape[1], d, page)
        pool = pool.astype(_i)
        a, b, e = page * d // 2, page * (d // 2 + d // 32), page * (d + d // 32)
        kb = pool[..., :a].reshape(*pool.shape[:2], page, d // 2)
        vb = pool[..., b:e].reshape(*pool.shape[:2], page, d // 2)
        c.ks = pool[..., a:b].reshape(*pool.shape[:2], page, d // 32).copy()
        c.vs = pool[..., e:].copy()
        for ch in range(d):
            g, w = divmod(ch, 32)
            half, w = divmod(w, 16)
            byte = kb[..., 4 * (d // 32 * (w // 4) + g) + w % 4]
            c.kc[..., ch] = (byte >> (4 * half) & 15) - 8
            c.vc[..., ch] = (vb[..., ch % (d // 2)] >> (4 * (ch // (d // 2))) & 15) - 8
        return c

    def to_bytes(self):
        pages, heads, page, d = self.kc.shape
        kb, vb = np.zeros((pages, heads, page, d // 2), _i), np.zeros((pages, heads, page, d // 2), _i)
        for ch in range(d):
            g, w = divmod(ch, 32)
            half, w = divmod(w, 16)
            kb[..., 4 * (d // 32 * (w // 4) + g) + w % 4] |= (self.kc[..., ch] + 8) << (4 * half)
            vb[..., ch % (d // 2)] |= (self.vc[..., ch] + 8) << (4 * (ch // (d // 2)))
        flat = [t.reshape(pages, heads, -1) for t in (kb, self.ks, vb, self.vs)]
        return np.concatenate(flat, -1).astype(np.uint8)

    def append(self, k, v, slots):
        heads, d = self.kc.shape[1], self.d
        for t, slot in enumerate(slots):
            if slot < 0 or slot >= self.kc.shape[0] * self.page:
                continue
            p, o = divmod(int(slot), self.page)
            for h in range(heads):
                x = k[t, h * d:(h + 1) * d].astype(_i).reshape(-1, 32)
                self.kc[p, h, o], self.ks[p, h, o] = [a.reshape(-1) for a in _quantise(x)]
                c, s = _quantise(v[t, h * d:(h + 1) * d].astype(_i)[None])
                self.vc[p, h, o], self.vs[p, h, o] = c[0], s[0, 0]

    def rows(self, table, n, h):
        """Keys and values of the first n tokens of a sequence: codes, steps, and which of them lie in the pool."""
        j = np.arange(n)
        p = np.asarray(table, _i)[j // self.page]
        ok = (p >= 0) & (p < self.kc.shape[0])
        p, o = np.where(ok, p, 0), j % self.page
        return self.kc[p, h, o], self.ks[p, h, o], self.vc[p, h, o], self.vs[p, h, o], ok


def _quantise(x):
    step = -(-8 * np.abs(x).max(-1, keepdims=True) // 7)
    return np.where(step > 0, (16 * x + step) // np.maximum(2 * step, 1), 0), step


def attention(cache, q, q_heads, q_start, lens, table, qk, I0, N, pv, out, weights=None):
    """Writes out (int64 copy of what it held) and returns (out, weights)."""
    heads, d = cache.kc.shape[1], cache.d
    G, z = q_heads // heads, (I0 << N).bit_length() - 8
    out = np.asarray(out, _i).copy()
    weights = None if weights is None else np.asarray(weights, _i).copy()
    for b, L in enumerate(lens):
        q0, q1, L = int(q_start[b]), int(q_start[b + 1]), int(L)
        for h in range(heads):
            kc, ks, vc, vs, ok = cache.rows(table[b], L, h)
            K = kc * np.repeat(ks, 32, -1)
            for r in range(q0, q1):
                seen = np.flatnonzero(ok & (np.arange(L) <= L - (q1 - q0) + (r - q0)))
                for g in range(G):
                    c0 = (h * G + g) * d
                    if len(seen) == 0:
                        out[r, c0:c0 + d] = 0
                        continue
                    s = np.clip(rq(K[seen] @ np.asarray(q[r, c0:c0 + d], _i), *qk), -128, 127)
                    e = shiftexp(s.max() - s, I0, N)
                    den = int(e.sum())
                    u = (e * vs[seen] + (1 << (z - 1))) >> z
                    num = u @ vc[seen]
                    t = np.array([(int(v) << (z + 5)) // den for v in num], _i)
                    out[r, c0:c0 + d] = np.clip(rq(t, *pv), -128, 127)
                    if weights is not None:
                        weights[b, h, seen] += (e << 24) // den
    return out, weights


def evict(cache, weights, lens, table, dst_table, ldw_out, keep, sinks, recent):
    """(kept, new_lens, weights_out, the cache's bytes afterwards)."""
    B, heads = weights.shape[:2]
    kept, wo = np.full((B, heads, keep), -1, _i), np.zeros((B, heads, ldw_out), _i)
    names = ("kc", "ks", "vc", "vs")
    old = {n: getattr(cache, n).copy() for n in names}
    for b, L in enumerate(lens):
        L = int(L)
        for h in range(heads):
            w = [int(v) for v in weights[b, h, :L]]
            stay = list(range(L))
            if L > keep:
                order = sorted(range(sinks, L - recent), key=lambda j: (-w[j], j))[:keep - sinks - recent]
                stay = sorted(list(range(sinks)) + order + list(range(L - recent, L)))
            for i, j in enumerate(stay):
                kept[b, h, i], wo[b, h, i] = j, w[j]
                sp, dp = int(table[b][j // cache.page]), int(dst_table[b][i // cache.page])
                for n in names:
                    getattr(cache, n)[dp, h, i % cache.page] = old[n][sp, h, j % cache.page]
    return kept, np.minimum(np.asarray(lens), keep), wo, cache.to_bytes()
