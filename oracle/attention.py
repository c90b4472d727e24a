"""Attention and the paged 8-bit cache from their formulas, on the CPU: scores, weights and sums in float64; the cache's
quantizer in the float32 operations that its definition names.  Tests only."""
import numpy as np

GROUP = 64
NONE, CAUSAL, PREFIX = 0, 1, 2


def slot(t):
    """Byte of token t's value code among the 64 of its group and channel."""
    return 16 * (t % 16 // 4) + 4 * (t // 16) + t % 4


def _one(q, k, v, scale, mask=NONE, prefix=0, cap=0.0, slopes=None, seen=None, reach=None):
    """One sequence, q [n, Hq, D], k, v [m, Hkv, D] (float64) -> (o [n, Hq, D], tolerance of a binary16 result [n, Hq, D]).

    The tolerance counts, with A = sum w |v| / sum w: binary16 weights (2^-11 relative; where they are subnormal 2^-25, with a largest weight of 2^7 or
    more 2^-32 of that one, in the sum of the values and in that of the weights, so twice; `reach` [m, Hkv]: what such an error is multiplied by, where that
    is more than |v| - over the cache 127 times the value scale) against fp32 sums, fp32 scores ((D + 16) roundings of 2^-24 of sum |q k|, and of the other terms; it enters the weights
    and their sum, so twice), and the result's own rounding."""
    n, Hq, D = q.shape
    m, Hkv = k.shape[0], k.shape[1]
    o, tol = np.zeros_like(q), np.full_like(q, 2.0 ** -25)
    if m == 0 or n == 0:
        return o, tol
    p = np.arange(n)[:, None] + (m - n)
    j = np.arange(m)[None, :]
    vis = np.ones((n, m), bool) if mask == NONE else (j <= p) | ((j < prefix) if mask == PREFIX else False)
    if seen is not None:
        vis = vis & seen[None, :]
    any_ = vis.any(1)
    for h in range(Hq):
        kh, vh = k[:, h // (Hq // Hkv)], v[:, h // (Hq // Hkv)]
        x = scale * (q[:, h] @ kh.T)
        size = abs(scale) * (np.abs(q[:, h]) @ np.abs(kh).T)
        if cap > 0:
            x = cap * np.tanh(x / cap)
            size = size + cap
        if slopes is not None:
            x = x - float(slopes[h]) * np.abs(p - j)
            size = size + abs(float(slopes[h])) * np.abs(p - j)
        x = np.where(vis, x, -np.inf)
        top = np.where(any_, x.max(1, initial=-np.inf), 0.0)[:, None]
        w = np.exp(x - top)
        l = np.where(any_, w.sum(1), 1.0)[:, None]
        o[:, h] = (w @ vh) / l
        A = (w @ np.abs(vh)) / l
        delta = ((D + 16) * 2.0 ** -24 * np.where(vis, size, 0.0).max(1) + 2.0 ** -21)[:, None]
        most = np.abs(vh).max(1) if reach is None else reach[:, h // (Hq // Hkv)]
        far = vis.sum(1)[:, None] * 2.0 ** -31 * np.where(vis, most[None], 0.0).max(1)[:, None] / l
        err = A * (2.0 ** -11 + 2 * delta) + far
        tol[:, h] = err + 2.0 ** -11 * (np.abs(o[:, h]) + err) + 2.0 ** -25
    return o, tol


def attention(q, k, v, cu_q, cu_k, scale, mask=NONE, prefix=None, cap=0.0, slopes=None):
    """Packed sequences: q [T, Hq, D], k, v [Tk, Hkv, D] -> (o, tolerance); rows of no sequence are NaN."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    o, tol = np.full_like(q, np.nan), np.full_like(q, np.nan)
    for b in range(len(cu_q) - 1):
        a, e, c, d = cu_q[b], cu_q[b + 1], cu_k[b], cu_k[b + 1]
        o[a:e], tol[a:e] = _one(q[a:e], k[c:d], v[c:d], scale, mask, 0 if prefix is None else int(prefix[b]), cap, slopes)
    return o, tol


class Cache:
    """The cache as numpy arrays in the documented storage order; `table` [B, max_pages]."""

    def __init__(self, kc, vc, ks, vs, table):
        self.kc, self.vc, self.ks, self.vs, self.table = (np.array(x) for x in (kc, vc, ks, vs, table))
        self.pages, self.heads, self.page, self.D = self.kc.shape
        self.S = self.page // self.ks.shape[2]

    def _where(self, b, j):
        e = j // self.page
        if e >= self.table.shape[1]:
            return None
        pg = int(self.table[b, e])
        return (pg, j % self.page) if 0 <= pg < self.pages else None

    def token(self, b, j):
        """(k codes, v codes, k scale, v scale) [Hkv, ...] of token j of sequence b, or None where its page is none."""
        w = self._where(b, j)
        if w is None:
            return None
        pg, at = w
        return (self.kc[pg, :, at], self.vc[pg, :, at // GROUP, :, slot(at % GROUP)], self.ks[pg, :, at // self.S], self.vs[pg, :, at // self.S])

    def sequence(self, b, n):
        """float64 k, v [n, Hkv, D] and which tokens are there."""
        k, v, seen = np.zeros((n, self.heads, self.D)), np.zeros((n, self.heads, self.D)), np.zeros(n, bool)
        for j in range(n):
            t = self.token(b, j)
            if t is None:
                continue
            seen[j] = True
            k[j] = t[0].astype(np.float64) * t[2].astype(np.float64)[:, None]
            v[j] = t[1].astype(np.float64) * t[3].astype(np.float64)[:, None]
        return k, v, seen

    def append(self, k, v, cu, lens, q=None, rot=None, pairs=False, pos=None):
        """The append's definition, float32 operation by operation; returns dict(q_out, k_out, v_out)."""
        f = np.float32
        T = k.shape[0]
        out = dict(q_out=None if q is None else np.full(q.shape, np.nan, np.float16), k_out=np.full(k.shape, np.nan, np.float16),
                   v_out=np.full(v.shape, np.nan, np.float16))
        for b in range(len(cu) - 1):
            n = cu[b + 1] - cu[b]
            first = int(lens[b]) - n
            blocks = {}
            for i in range(n):
                j = first + i
                if j < 0:
                    continue
                t = cu[b] + i
                p = j if pos is None else int(pos[t])
                turn = (lambda x: x.copy()) if rot is None else (lambda x: rotate(x, rot[min(max(p, 0), len(rot) - 1)], pairs))
                if q is not None:
                    out["q_out"][t] = turn(q[t])
                blocks.setdefault(j // self.S, []).append((j, t, turn(k[t]), v[t]))
            for rows in blocks.values():
                j0 = rows[0][0]
                for which, codes, scales, name in ((2, self.kc, self.ks, "k_out"), (3, self.vc, self.vs, "v_out")):
                    h = np.stack([r[which] for r in rows]).astype(f)                       # [rows, Hkv, D]
                    w = self._where(b, j0)
                    old = np.zeros(self.heads, f)
                    if w is not None and j0 % self.S:
                        old = scales[w[0], :, w[1] // self.S].copy()
                    alpha = np.maximum(old, np.abs(h).max((0, 2)) / f(127.0))
                    safe = np.where(alpha > 0, alpha, f(1.0))
                    c = np.clip(np.rint(h / safe[None, :, None]), -127, 127)
                    for x, r in zip(c, rows):
                        out[name][r[1]] = (x * safe[:, None]).astype(np.float16)
                    if w is None:
                        continue
                    for at in range(w[1] // self.S * self.S, w[1]):                      # earlier tokens of the block
                        was = self._codes(codes, w[0], at)
                        again = np.clip(np.rint(was.astype(f) * old[:, None] / safe[:, None]), -127, 127).astype(np.int8)
                        self._set(codes, w[0], at, np.where((alpha > old)[:, None], again, was))
                    scales[w[0], :, w[1] // self.S] = alpha
                    for x, r in zip(c, rows):
                        self._set(codes, w[0], self._where(b, r[0])[1], x.astype(np.int8))
        return out

    def _codes(self, codes, pg, at):
        return codes[pg, :, at].copy() if codes is self.kc else codes[pg, :, at // GROUP, :, slot(at % GROUP)].copy()

    def _set(self, codes, pg, at, x):
        if codes is self.kc:
            codes[pg, :, at] = x
        else:
            codes[pg, :, at // GROUP, :, slot(at % GROUP)] = x


def rotate(x, row, pairs):
    """x [H, D] binary16, row [rot_dim / 2, 2] float32 (cos, sin): each operation rounded to float32, the result to binary16."""
    f = np.float32
    half = row.shape[0]
    y = x.astype(f)
    i = 2 * np.arange(half) if pairs else np.arange(half)
    j = i + 1 if pairs else i + half
    a, b, c, s = y[:, i], y[:, j], row[:, 0].astype(f), row[:, 1].astype(f)
    out = y.copy()
    out[:, i] = a * c - b * s
    out[:, j] = b * c + a * s
    return out.astype(np.float16)


def attention_cached(q, cache, cu_q, lens, scale, mask=CAUSAL, prefix=None, cap=0.0, slopes=None):
    q = np.asarray(q, np.float64)
    o, tol = np.full_like(q, np.nan), np.full_like(q, np.nan)
    for b in range(len(cu_q) - 1):
        k, v, seen = cache.sequence(b, int(lens[b]))
        reach = np.zeros((len(seen), cache.heads))
        for j in np.flatnonzero(seen):
            reach[j] = 127.0 * cache.token(b, j)[3]
        a, e = cu_q[b], cu_q[b + 1]
        o[a:e], tol[a:e] = _one(q[a:e], k, v, scale, mask, 0 if prefix is None else int(prefix[b]), cap, slopes, seen, reach)
    return o, tol
