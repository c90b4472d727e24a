"""The layers in 8-bit floating point, routing and the experts' layers in float64 (numpy), from their formulas, with the tolerances that their roundings give.
Used by the tests only.

Roundings: fp32 is off by at most 2^-24 of a value, fp16 by 2^-11 (2^-25 among its subnormals), e4m3 by half a step.  The matrix cores' sums of a
block are allowed one truncation (2^-23) for each addition.
"""
import numpy as np

BLOCK = 128


def blocks(n):
    return -(-n // BLOCK)


def _step(v):
    """The distance between neighbouring e4m3 values at v."""
    _, e = np.frexp(np.abs(v))
    return np.exp2(np.maximum(e - 1.0, -6.0) - 3.0)


def e4m3(v):
    """The nearest e4m3 value, ties to even."""
    v = np.asarray(v, np.float64)
    step = _step(v)
    return np.clip(np.rint(v / step) * step, -448.0, 448.0)


def decode(codes):
    """uint8 codes -> values."""
    c = np.asarray(codes, np.uint8).astype(np.int64)
    s, e, m = c >> 7, (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    return np.where(s == 1, -v, v)


def silu(a):
    return a / (1.0 + np.exp(-a))


def by_block(s, n):
    """One scale for every channel."""
    return np.repeat(s, BLOCK, axis=-1)[..., :n]


def block_max(v):
    K = v.shape[-1]
    pad = np.zeros(v.shape[:-1] + (blocks(K) * BLOCK,))
    pad[..., :K] = np.abs(v)
    return pad.reshape(v.shape[:-1] + (blocks(K), BLOCK)).max(-1)


def quantize(v):
    """float64 [..., K] -> the exact quotients 448 v / amax, their codes' values, and the scales in fp32."""
    amax = block_max(v)
    scales = np.where(amax > 0, amax.astype(np.float32) / np.float32(448.0), np.float32(1.0)).astype(np.float32)
    t = 448.0 * v / by_block(np.where(amax > 0, amax, 1.0), v.shape[-1])
    return t, e4m3(t), scales


def product(c, s, w, sw, bias=None, core=False):
    """Codes' values c [M,K], scales s [M,KB], w [N,K], sw [NB,KB] -> (u [M,N], how far fp32 may be from it).  core: the matrix cores' sums of codes, which cut
    each of 8 neighbouring products off below 2^-13 of the power of two that their largest reaches: 8 * 2^-13 of the largest, which is at most the product of
    the largest factors."""
    K, N = c.shape[-1], w.shape[0]
    wide = np.repeat(by_block(sw.astype(np.float64), K), BLOCK, axis=0)[:N] * w
    x = c * by_block(s.astype(np.float64), K)
    u = x @ wide.T
    tol = (K + 3 * blocks(K)) * 2.0 ** -23 * (np.abs(x) @ np.abs(wide).T)
    if core:
        tol = tol + 2.0 ** -10 * (np.abs(x).reshape(x.shape[0], K // 8, 8).max(-1) @ np.abs(wide).reshape(N, K // 8, 8).max(-1).T)
    if bias is not None:
        u = u + bias.astype(np.float64)
        tol = tol + 2.0 ** -24 * np.abs(u)
    return u, tol


def half_step(u):
    return np.maximum(np.abs(u) * 2.0 ** -11, 2.0 ** -25)


def row_step(o):
    """How far a row's output may be off by its rounding: binary16's half step, of 64 neighbours that reach 2^15 with the exponent that takes the largest of them
    below 2^15 again: then the subnormals' half step, 2^-25, counts as many times as much."""
    N = o.shape[-1]
    pad = np.zeros(o.shape[:-1] + (-(-N // 64) * 64,))
    pad[..., :N] = np.abs(o)
    _, e = np.frexp(pad.reshape(o.shape[:-1] + (-1, 64)).max(-1))
    return np.maximum(np.abs(o) * 2.0 ** -11, np.repeat(np.exp2(np.maximum(e - 15, 0) - 25.0), 64, axis=-1)[..., :N])


def gelu(u):
    return u / (1.0 + np.exp(-2.0 * np.sqrt(2.0 / np.pi) * (u + 0.044715 * u ** 3)))


def layer(c, s, w, sw, bias=None, act=0, residual=None, gate=None, gate_rows=1, core=False):
    """(y, tolerance) of qgemm_f8 before the last rounding, that rounding in the tolerance."""
    u, tol = product(c, s, w, sw, bias, core)
    if act:
        # |gelu'| <= 1.13; an exponent of up to 30 (2^-30 is nothing) is off by 30 * 2^-23 ln 2 < 2^-18
        u, tol = gelu(u), 1.13 * tol + 2.0 ** -18 * np.abs(gelu(u)) + 2.0 ** -29
    if residual is not None or gate is not None:
        tol = tol + half_step(np.abs(u) + tol)
        g = np.ones_like(u) if gate is None else np.repeat(gate.astype(np.float64), gate_rows, axis=0)
        u, tol = g * u + (0.0 if residual is None else residual.astype(np.float64)), np.abs(g) * tol
        tol = tol + 2.0 ** -24 * np.abs(u)
    return u, tol + half_step(np.abs(u) + tol)


def route(logits, k, bias=None, sigmoid=False, groups=1, top_groups=1, group_top=2, renorm=True, scale=1.0):
    """(ids [T,k], weights [T,k]) token by token."""
    most = float(np.finfo(logits.dtype).max)
    T, E = logits.shape
    ids, weights = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        x = logits[t].astype(np.float64)
        x = np.where(np.isnan(x), -np.inf, np.minimum(x, most))
        alive = x > -np.inf
        if not alive.any():
            continue
        with np.errstate(over="ignore"):
            s = 1.0 / (1.0 + np.exp(-x)) if sigmoid else np.exp(x - x.max()) / np.exp(x - x.max()).sum()
        s[~alive] = 0.0
        c = s if bias is None else s + bias.astype(np.float64)
        alive &= ~np.isnan(c) & (c > -np.inf)
        if groups > 1:
            worth = []
            for g in range(groups):
                part = slice(g * (E // groups), (g + 1) * (E // groups))
                best = np.sort(c[part][alive[part]])[::-1][:group_top]
                worth.append(best.sum() if best.size else -np.inf)
            kept = [g for g in np.argsort(-np.array(worth), kind="stable")[:top_groups] if worth[g] > -np.inf]
            alive &= np.isin(np.arange(E) // (E // groups), kept)
        key = np.where(alive, x if bias is None else c, -np.inf)
        order = [e for e in np.argsort(-key, kind="stable")[:k] if alive[e]]
        w = s[order]
        if renorm and w.sum() > 0:
            w = w / w.sum()
        ids[t, :len(order)], weights[t, :len(order)] = order, w * scale
    return ids, weights


def gated(g, u, dg, du):
    """silu(g) * u and how far it may be off, where g and u are off by dg and du."""
    h = silu(g) * u
    return h, 1.1 * dg * (np.abs(u) + du) + np.abs(silu(g)) * du + 2.0 ** -20 * np.abs(h) + 2.0 ** -110


def quantized(h, dh):
    """What the codes and scales of h stand for, and how far that may be off where h is off by dh: a code whose quotient lies as near to the middle
    of two of them as that may be the other one."""
    K = h.shape[-1]
    t, c, s = quantize(h)
    amax = by_block(np.maximum(block_max(h), 1e-300), K)
    damax = by_block(block_max(dh), K)
    dt = 448.0 * (dh / amax + np.abs(h) / amax * (damax / amax)) + 2.0 ** -22 * np.abs(t)
    size = np.abs(t)
    step = _step(size)
    near = np.abs(size - (np.floor(size / step) + 0.5) * step) <= dt
    scale = by_block(s.astype(np.float64), K)
    off = np.where(near, step + dt, 0.0) * scale
    return c, s, off + np.abs(c) * scale * (damax / amax + 2.0 ** -22)


def experts(x, ids, weights, w_up, up_scale, w_down, down_scale, residual=None):
    """(y, tolerance) of experts_f8; w_up [E,2,I,K] and w_down [E,N,I] are the codes' values."""
    T, N = x.shape[0], w_down.shape[1]
    I = w_down.shape[2]
    y = np.zeros((T, N)) if residual is None else residual.astype(np.float64)
    size, tol = np.abs(y), np.zeros((T, N))
    _, c, s = quantize(x.astype(np.float64))
    for e in range(w_down.shape[0]):
        t, j = np.nonzero(ids == e)
        if not t.size:
            continue
        g, dg = product(c[t], s[t], w_up[e, 0], up_scale[e, 0])
        u, du = product(c[t], s[t], w_up[e, 1], up_scale[e, 1])
        h, dh = gated(g, u, dg, du)
        hc, hs, dhq = quantized(h, dh)
        o, do = product(hc, hs, w_down[e], down_scale[e])
        wide = np.abs(np.repeat(by_block(down_scale[e].astype(np.float64), I), BLOCK, axis=0)[:N] * w_down[e])
        do = do + dhq @ wide.T
        do = do + row_step(np.abs(o) + do)
        w = weights[t, j].astype(np.float64)[:, None]
        np.add.at(y, t, w * o)
        np.add.at(size, t, np.abs(w * o))
        np.add.at(tol, t, np.abs(w) * do)
    tol = tol + (ids.shape[1] + 1) * 2.0 ** -24 * (size + tol)
    return y, tol + half_step(np.abs(y) + tol)
