"""attention_f16, daq_kv_append and attention_kv8 against the 64-bit oracle, through the C ABI.  The tolerance of every attention output is
the oracle's own count of roundings (oracle/attention.py); cache codes, scales, rotated rows and returned values are compared bit for bit."""
import numpy as np
import pytest
import torch

import paper_2511_11446_amd as ql
from oracle import attention as oa

pytestmark = pytest.mark.gpu


def _rng(*key):
    return np.random.default_rng([1511, *key])


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _dev(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _f16(g, *shape, size=1.0):
    return (g.standard_normal(shape, dtype=np.float32) * np.float32(size)).astype(np.float16)


def _close(o, ref, tol, name=""):
    o = o.cpu().numpy().astype(np.float64)
    live = ~np.isnan(ref)
    bad = ~(np.abs(o - ref) <= tol) & live
    assert not bad.any(), "%s: %d of %d off, worst %.3g times the tolerance at %s" % (
        name, bad.sum(), live.sum(), np.nanmax(np.where(live, np.abs(o - ref) / tol, 0)), np.argwhere(bad)[:3].tolist())


def _dense(key, nq, nk, Hq, Hkv, D, mask=0, cap=0.0, slopes=False, fused=False, equal=False, size=1.0, extra=0):
    """Runs one case; nq / nk: lengths of the sequences; extra: rows behind the last one."""
    g = _rng(*key)
    Tq, Tk = sum(nq) + extra, sum(nk) + extra
    if fused:
        rows = _f16(g, Tq, (Hq + 2 * Hkv) * D, size=size)
        d = _dev(rows)
        q, k, v = rows[:, :Hq * D].reshape(Tq, Hq, D), rows[:, Hq * D:(Hq + Hkv) * D].reshape(Tq, Hkv, D), rows[:, (Hq + Hkv) * D:].reshape(Tq, Hkv, D)
        dq, dk, dv = d[:, :Hq * D].unflatten(1, (Hq, D)), d[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D)), d[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
    else:
        q, k, v = _f16(g, Tq, Hq, D, size=size), _f16(g, max(Tk, 1), Hkv, D, size=size), _f16(g, max(Tk, 1), Hkv, D, size=size)
        dq, dk, dv = _dev(q), _dev(k), _dev(v)
    prefix = g.integers(0, max(max(nk), 1) + 2, len(nq)).astype(np.int32) if mask == 2 else None
    sl = g.uniform(0, 0.3, Hq).astype(np.float32) if slopes else None
    cq, ck = _cu(nq), _cu(nk)
    scale = D ** -0.5
    ref, tol = oa.attention(q, k, v, cq, ck, scale, mask, prefix, cap, sl)
    o = torch.full((Tq, Hq, D), 7.0, dtype=torch.float16, device="cuda")
    am = torch.full((Tq,), -1, dtype=torch.int32, device="cuda")
    out = ql.attention_f16(dq, dk, dv, batch=len(nq), cu_q=None if equal else _dev(cq), cu_k=None if equal else _dev(ck), mask=mask, prefix=_dev(prefix),
                           cap=cap, slopes=_dev(sl), o=o, row_absmax=am)
    torch.cuda.synchronize()
    assert out is o
    _close(o, ref, tol, str(key))
    assert bool((o[cq[-1]:] == 7.0).all()), "rows behind the last sequence changed"
    if sum(nq):
        want = o[:cq[-1]].abs().flatten(1).amax(1).view(torch.int16).int()
        assert torch.equal(am[:cq[-1]], want), "row maxima"
    return o


@pytest.mark.parametrize("D", [8, 16, 24, 32, 40, 64, 72, 80, 96, 104, 128, 136, 192, 200, 256])
def test_head_sizes(D):
    _dense((1, D), [70, 33], [70, 33], 2, 2, D, fused=True)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500])
@pytest.mark.parametrize("mask", [0, 1, 2])
def test_lengths_and_masks(n, mask):
    _dense((2, n, mask), [n], [n], 2, 1, 64, mask=mask)


@pytest.mark.parametrize("nq, nk", [([1], [1000]), ([1, 1, 1], [1, 700, 64]), ([5, 0, 17], [300, 40, 5]), ([40], [7]), ([3, 64, 100], [0, 64, 1]),
                                    ([0, 0, 9], [4, 0, 130])])
@pytest.mark.parametrize("mask", [0, 1, 2])
def test_rows_and_keys_of_different_number(nq, nk, mask):
    """Causal rows in front of the first key, sequences without keys or rows: their outputs are zero, others are right."""
    _dense((3, sum(nq), sum(nk), mask), nq, nk, 4, 2, 72, mask=mask)


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (3, 1), (6, 2), (8, 1), (12, 4), (5, 5), (40, 2), (7, 7)])
def test_shared_key_heads(Hq, Hkv):
    _dense((4, Hq, Hkv), [37, 90, 4], [37, 90, 4], Hq, Hkv, 64, mask=1, fused=True)


@pytest.mark.parametrize("cap, slopes", [(30.0, False), (0.0, True), (5.0, True)])
@pytest.mark.parametrize("mask", [0, 1, 2])
def test_score_forms(cap, slopes, mask):
    _dense((5, int(cap), slopes, mask), [150, 61], [150, 61], 4, 2, 128, mask=mask, cap=cap, slopes=slopes, size=2.0)


@pytest.mark.parametrize("cap", [2.0 ** -10, 2.0 ** 10])
def test_smallest_and_largest_cap(cap):
    """The oracle's tolerance has (D + 16) 2^-24 of the cap; the capped score is off by about 2^-22 of it."""
    _dense((13, int(cap)), [70, 9], [130, 40], 2, 1, 64, mask=1, cap=cap, size=2.0)
    _cached((43, int(cap)), [1, 2], [200, 70], 4, 2, 64, 64, 16, cap=cap)
    _cached((44, int(cap)), [90, 70], [200, 70], 4, 2, 64, 64, 64, cap=cap)


def test_rows_behind_the_last_sequence_stay():
    _dense((6,), [20, 30], [64, 3], 3, 3, 40, extra=9)


def test_equal_lengths_need_no_first_rows():
    _dense((7,), [64] * 5, [64] * 5, 4, 4, 72, equal=True, fused=True)
    _dense((7, 1), [16] * 3, [200] * 3, 4, 4, 64, equal=True)


@pytest.mark.parametrize("size", [0.01, 8.0, 40.0])
def test_small_and_large_scores(size):
    """Weights that are nearly alike, and rows where one key takes everything; the maximum grows along the keys."""
    _dense((8, int(size * 100)), [130], [333], 2, 2, 64, size=size)


def test_growing_maximum():
    """Every later key has the larger score, by more than what one weight can hold."""
    D, n = 64, 256
    q = torch.ones((1, 1, D), dtype=torch.float16, device="cuda")
    k = (torch.arange(n, device="cuda").float() * 0.75).half()[:, None, None].expand(n, 1, D).contiguous()
    v = _dev(_f16(_rng(9), n, 1, D))
    for order in (torch.arange(n), torch.arange(n).flip(0), torch.randperm(n, generator=torch.Generator().manual_seed(3))):
        kk, vv = k[order.cuda()].contiguous(), v[order.cuda()].contiguous()
        ref, tol = oa.attention(q.cpu().numpy(), kk.cpu().numpy(), vv.cpu().numpy(), [0, 1], [0, n], 1.0)
        o = ql.attention_f16(q, kk, vv, scale=1.0)
        torch.cuda.synchronize()
        _close(o, ref, tol)


def test_heads_first_and_shared_rows():
    """[H, T, D] storage, and keys that every head reads from the same place (stride 0)."""
    g = _rng(10)
    T, H, D = 100, 3, 64
    q, k, v = _f16(g, H, T, D), _f16(g, T, 1, D), _f16(g, H, T, D)
    dq, dv = _dev(q).transpose(0, 1), _dev(v).transpose(0, 1)
    dk = _dev(k).expand(T, H, D)
    o = torch.empty((H, T, D), dtype=torch.float16, device="cuda").transpose(0, 1)
    ql.attention_f16(dq, dk, dv, o=o)
    torch.cuda.synchronize()
    ref, tol = oa.attention(q.transpose(1, 0, 2), np.repeat(k, H, 1), v.transpose(1, 0, 2), [0, T], [0, T], D ** -0.5)
    _close(o, ref, tol)


def test_values_outside_the_sequences_do_not_count():
    """NaN and infinities in rows of no sequence, next to rows that count."""
    g = _rng(11)
    D, H = 72, 2
    q, k, v = _f16(g, 60, H, D), _f16(g, 100, H, D), _f16(g, 100, H, D)
    cq, ck = np.array([3, 20, 41], np.int32), np.array([10, 43, 77], np.int32)
    for x, lo, hi in ((q, 3, 41), (k, 10, 77), (v, 10, 77)):
        x[:lo], x[hi:] = np.nan, np.inf
    o = torch.full((60, H, D), 3.0, dtype=torch.float16, device="cuda")
    ql.attention_f16(_dev(q), _dev(k), _dev(v), cu_q=_dev(cq), cu_k=_dev(ck), o=o, mask=1)
    torch.cuda.synchronize()
    ref, tol = oa.attention(q, k, v, cq, ck, D ** -0.5, 1)
    _close(o, ref, tol)
    assert bool((o[:3] == 3.0).all()) and bool((o[41:] == 3.0).all())


# ---- the cache ------------------------------------------------------------------------------------------------------------------

class _Cached:
    """A cache with random codes and scales, pages in no order, on both sides."""

    def __init__(self, g, B, most, Hkv, D, page, S, spare=2):
        self.B, self.page = B, page
        per = -(-most // page)
        P = B * per + spare
        kc = g.integers(-127, 128, (P, Hkv, page, D)).astype(np.int8)
        vc = g.integers(-127, 128, (P, Hkv, page // 64, D, 64)).astype(np.int8)
        ks, vs = (g.uniform(0.005, 0.03, (P, Hkv, page // S)).astype(np.float32) for _ in range(2))
        table = g.permutation(P)[:B * per].reshape(B, per).astype(np.int32)
        self.ref = oa.Cache(kc, vc, ks, vs, table)
        self.dev = ql.KvCache8(_dev(kc), _dev(vc), _dev(ks), _dev(vs))
        self.table = _dev(table)

    def same(self):
        torch.cuda.synchronize()
        for name, a, b in (("k", self.dev.k, self.ref.kc), ("v", self.dev.v, self.ref.vc), ("k_scale", self.dev.k_scale, self.ref.ks),
                           ("v_scale", self.dev.v_scale, self.ref.vs)):
            a = a.cpu().numpy()
            assert np.array_equal(a, b), "%s: %d of %d differ, first at %s" % (name, (a != b).sum(), a.size, np.argwhere(a != b)[:2].tolist())


def _append(g, c, lens, nq, Hq, rot=None, pairs=False, pos=None, size=1.0, equal=False, values=True):
    Hkv, D = c.ref.heads, c.ref.D
    T = sum(nq)
    cu = _cu(nq)
    rows = _f16(g, T, (Hq + 2 * Hkv) * D, size=size)
    q, k, v = rows[:, :Hq * D].reshape(T, Hq, D), rows[:, Hq * D:(Hq + Hkv) * D].reshape(T, Hkv, D), rows[:, (Hq + Hkv) * D:].reshape(T, Hkv, D)
    d = _dev(rows)
    dq, dk, dv = d[:, :Hq * D].unflatten(1, (Hq, D)), d[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D)), d[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
    ref = c.ref.append(k, v, cu, lens, q, rot, pairs, pos)
    q_out = torch.full((T, Hq, D), 5.0, dtype=torch.float16, device="cuda")
    k_out, v_out = (torch.full((T, Hkv, D), 5.0, dtype=torch.float16, device="cuda") if values else None for _ in range(2))
    ql.daq_kv_append(c.dev, dk, dv, c.table, _dev(np.asarray(lens, np.int32)), cu=None if equal else _dev(cu), q=dq, rot=_dev(rot), rot_pairs=pairs,
                     pos=_dev(pos), q_out=q_out, k_out=k_out, v_out=v_out)
    c.same()
    for name, t in (("q_out", q_out), ("k_out", k_out), ("v_out", v_out)):
        if t is None:
            continue
        a, b = t.cpu().numpy(), ref[name]
        live = ~np.isnan(b)
        assert np.array_equal(a[live], b[live]), name
        assert (a[~live] == 5.0).all(), name
    return q_out


def _table(rows, rot_dim):
    a = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(rot_dim // 2) / (rot_dim // 2))
    return np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)


@pytest.mark.parametrize("S", [1, 16, 32, 64])
@pytest.mark.parametrize("D, page", [(64, 64), (72, 128), (128, 64), (256, 192), (8, 64)])
def test_append_prompts_then_tokens(S, D, page):
    """Prompts that end inside groups, then single tokens and short runs that raise the scales of blocks with earlier tokens."""
    g = _rng(20, S, D, page)
    c = _Cached(g, 3, 400, 2, D, page, S)
    rot = _table(400, D // 16 * 16) if D >= 16 else None
    lens = np.array([70, 1, 191], np.int32)
    _append(g, c, lens, [70, 1, 191], 4, rot, size=0.5)
    for n, size in ((1, 0.4), (1, 3.0), (3, 1.0), (1, 5.0), (20, 2.0), (65, 6.0), (1, 0.1)):
        lens = lens + n
        _append(g, c, lens, [n] * 3, 4, rot, size=size, equal=n == 1)


def test_append_ragged_runs_and_sequences_without_tokens():
    g = _rng(21)
    c = _Cached(g, 70, 300, 1, 64, 64, 16)
    nq = [int(x) for x in g.integers(0, 40, 70)]
    lens = np.array([n + int(x) for n, x in zip(nq, g.integers(0, 250, 70))], np.int32)
    _append(g, c, lens, nq, 3, _table(300, 32), pairs=True)


@pytest.mark.parametrize("pairs", [False, True])
def test_append_rotation_by_given_positions(pairs):
    g = _rng(22, pairs)
    c = _Cached(g, 2, 128, 2, 96, 64, 32)
    pos = g.integers(-2, 60, 50).astype(np.int32)          # some outside the table: its nearest row
    _append(g, c, np.array([30, 20], np.int32), [30, 20], 2, _table(50, 64), pairs, pos)


def test_append_zero_blocks():
    """A block of zeros has scale 0; a later token raises it."""
    g = _rng(23)
    c = _Cached(g, 1, 64, 1, 64, 64, 64)
    _append(g, c, np.array([5], np.int32), [5], 1, size=0.0)
    assert float(c.dev.k_scale[c.table[0, 0].item()].max()) == 0.0
    _append(g, c, np.array([6], np.int32), [1], 1, size=0.01)
    _append(g, c, np.array([7], np.int32), [1], 1, size=0.0)
    _append(g, c, np.array([40], np.int32), [33], 1, size=1.0)


def test_append_to_pages_that_are_none():
    """Entries outside the pool, and tokens behind the table's end or in front of the sequence: nothing is written for them."""
    g = _rng(24)
    c = _Cached(g, 4, 192, 2, 64, 64, 32)
    for b, e, bad in ((0, 1, -1), (1, 0, 10 ** 6), (3, 2, c.ref.pages)):
        c.ref.table[b, e] = bad
    c.table.copy_(torch.from_numpy(c.ref.table))
    _append(g, c, np.array([100, 70, 230, 190], np.int32), [100, 70, 90, 100], 2, _table(300, 64))
    _append(g, c, np.array([5, 70, 192, 190], np.int32), [9, 1, 1, 1], 2, _table(300, 64))


def _cached(key, nq, nk, Hq, Hkv, D, page=64, S=64, mask=1, cap=0.0, slopes=False, equal=False, cache=None, size=1.0):
    g = _rng(*key)
    c = cache or _Cached(g, len(nq), max(max(nk), 1), Hkv, D, page, S)
    T = sum(nq)
    q = _f16(g, T, Hq, D, size=size)
    prefix = g.integers(0, max(nk) + 2, len(nq)).astype(np.int32) if mask == 2 else None
    sl = g.uniform(0, 0.3, Hq).astype(np.float32) if slopes else None
    cu = _cu(nq)
    scale = 0.5 * D ** -0.5
    ref, tol = oa.attention_cached(q, c.ref, cu, nk, scale, mask, prefix, cap, sl)
    am = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    o = ql.attention_kv8(_dev(q), c.dev, c.table, _dev(np.asarray(nk, np.int32)), cu_q=None if equal else _dev(cu), mask=mask, prefix=_dev(prefix), scale=scale,
                         cap=cap, slopes=_dev(sl), row_absmax=am)
    torch.cuda.synchronize()
    _close(o, ref, tol, str(key))
    assert torch.equal(am, o.abs().flatten(1).amax(1).view(torch.int16).int()), "row maxima"
    return o


@pytest.mark.parametrize("S", [1, 16, 32, 64])
@pytest.mark.parametrize("D", [8, 32, 40, 64, 72, 96, 128, 160, 192, 256])
def test_cached_tokens(S, D):
    _cached((30, S, D), [1, 1, 1], [1, 64, 333], 8, 2, D, 64, S, equal=True)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 1000, 2500])
def test_cached_lengths(n):
    _cached((31, n), [1], [n], 4, 1, 128, 128, 32, equal=True)


@pytest.mark.parametrize("Hq, Hkv", [(1, 1), (2, 2), (3, 1), (8, 1), (16, 1), (17, 1), (32, 1), (40, 1), (12, 4)])
@pytest.mark.parametrize("n", [1, 4, 9])
def test_cached_rows_per_key_head(Hq, Hkv, n):
    """From one packed row to hundreds for a key head."""
    _cached((32, Hq, Hkv, n), [n, n], [200, n], Hq, Hkv, 64, 64, 16, equal=True)


@pytest.mark.parametrize("mask", [0, 1, 2])
@pytest.mark.parametrize("cap, slopes", [(0.0, False), (20.0, True)])
def test_cached_chunks(mask, cap, slopes):
    _cached((33, mask, int(cap)), [130, 1, 64, 0, 200], [500, 1, 64, 70, 200], 4, 2, 64, 64, 32, mask, cap, slopes)


def test_cached_sequences_without_tokens_and_rows_in_front():
    _cached((34,), [1, 3, 2, 40], [0, 2, 100, 9], 4, 2, 64, 64, 64)


def test_cached_many_sequences():
    g = _rng(35)
    nk = [int(x) for x in g.integers(1, 400, 150)]
    _cached((35, 1), [1] * 150, nk, 4, 2, 64, 64, 64, equal=True)


def test_cached_scales_of_very_different_size():
    """Values whose scales differ by ten powers of two within a sequence: small ones still count where their weight is large."""
    g = _rng(36)
    for S in (1, 32):
        c = _Cached(g, 2, 300, 2, 64, 64, S)
        c.ref.vs[:] = (c.ref.vs * 2.0 ** g.integers(-10, 11, c.ref.vs.shape)).astype(np.float32)
        c.dev.v_scale.copy_(torch.from_numpy(c.ref.vs))
        _cached((36, S), [1, 1], [300, 170], 4, 2, 64, 64, S, equal=True, cache=c)


def test_cached_pages_that_are_none_are_not_visible():
    g = _rng(37)
    c = _Cached(g, 3, 256, 2, 64, 64, 32)
    for b, e, bad in ((0, 1, -1), (1, 0, 10 ** 6), (2, 0, -5), (2, 1, c.ref.pages), (2, 2, -1), (2, 3, -1)):
        c.ref.table[b, e] = bad
    c.table.copy_(torch.from_numpy(c.ref.table))
    o = _cached((37, 1), [1, 70, 3], [256, 256, 256], 4, 2, 64, 64, 32, cache=c)
    assert bool((o[71:] == 0).all())


def test_cached_scales_behind_the_end_do_not_count():
    """Scales of tokens that are not there hold anything."""
    g = _rng(38)
    for S in (1, 16, 64):
        c = _Cached(g, 2, 128, 1, 64, 64, S)
        used = {(int(c.ref.table[b, j // 64]), j % 64 // S) for b, n in ((0, 70), (1, 3)) for j in range(n)}
        for p in range(c.ref.pages):
            for i in range(64 // S):
                if (p, i) not in used:
                    c.ref.ks[p, :, i] = np.nan
                    c.ref.vs[p, :, i] = np.inf
        c.dev.k_scale.copy_(torch.from_numpy(c.ref.ks))
        c.dev.v_scale.copy_(torch.from_numpy(c.ref.vs))
        _cached((38, S), [1, 1], [70, 3], 2, 1, 64, 64, S, equal=True, cache=c)


@pytest.mark.parametrize("S", [1, 16, 64])
@pytest.mark.parametrize("D", [8, 32, 40, 72, 88, 96, 128, 136, 200, 256])
def test_cached_chunks_of_every_head_size(S, D):
    """Many rows: the cache's codes become tiles."""
    _cached((39, S, D), [150, 90], [400, 91], 4, 2, D, 64, S)


def test_cached_chunks_over_long_sequences_are_cut():
    """Few tiles over many keys: parts of the keys, joined."""
    _cached((40,), [70, 3], [3001, 1500], 4, 1, 64, 128, 32, cap=30.0, slopes=True)


def test_cached_tokens_with_pages_that_are_none():
    """The same for single tokens: whole sequences without a page, and a page missing in the middle of one."""
    g = _rng(41)
    c = _Cached(g, 4, 640, 2, 128, 64, 32)
    c.ref.table[0, 3:7] = -1
    c.ref.table[1, :] = 10 ** 6
    c.ref.table[2, 0], c.ref.table[2, 9] = c.ref.pages, -7
    c.table.copy_(torch.from_numpy(c.ref.table))
    o = _cached((41, 1), [1, 2, 3, 1], [640, 640, 600, 64], 4, 2, 128, 64, 32, cache=c)
    assert bool((o[1:3] == 0).all())


def test_few_rows_over_long_keys_are_cut():
    _dense((12,), [1], [9001], 2, 1, 64, mask=1)
    _dense((12, 1), [33, 2], [2000, 3000], 2, 2, 72, mask=2, cap=30.0, slopes=True)
    _dense((12, 2), [20], [2500], 4, 1, 200)


def test_offsets_past_two_gigabytes():
    """Pages at the end of a cache whose keys alone hold more than 2^31 codes."""
    Hkv, D, page = 4, 128, 64
    P = (1 << 31) // (Hkv * D * page) + 40
    cache = ql.KvCache8.empty(P, Hkv, D, page=page, scale_tokens=64)
    g = _rng(42)
    n = 130
    table = np.array([[P - 1, 3, P - 17]], np.int32)
    x = _f16(g, n, 3 * Hkv * D)
    q, k, v = (x[:, i * Hkv * D:(i + 1) * Hkv * D].reshape(n, Hkv, D) for i in range(3))
    dx = _dev(x)
    dq, dk, dv = (dx[:, i * Hkv * D:(i + 1) * Hkv * D].unflatten(1, (Hkv, D)) for i in range(3))
    k_out, v_out = (torch.empty((n, Hkv, D), dtype=torch.float16, device="cuda") for _ in range(2))
    lens = _dev(np.array([n], np.int32))
    ql.daq_kv_append(cache, dk, dv, _dev(table), lens, k_out=k_out, v_out=v_out)
    one = ql.attention_kv8(dq[-1:], cache, _dev(table), lens)
    many = ql.attention_kv8(dq, cache, _dev(table), lens)
    torch.cuda.synchronize()
    pages = [int(p) for p in table[0]]
    kc = cache.k[pages].cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, Hkv, D)[:n].astype(np.float64)
    ks = cache.k_scale[pages].cpu().numpy()[:, :, 0].repeat(64, 0)[:n].astype(np.float64)
    # a code is the rounded 32-bit quotient h / s, below 128 and so off by at most 2^-18 before it is rounded: half a step and 2^-18 of it
    assert (np.abs(kc * ks[..., None] - k) <= (0.5 + 2.0 ** -18) * ks[..., None]).all(), "keys at the end of the pool"
    order = [oa.slot(t) for t in range(64)]
    vc = cache.v[pages].cpu().numpy()[:, :, 0][..., order].transpose(0, 3, 1, 2).reshape(-1, Hkv, D)[:n].astype(np.float64)
    vs = cache.v_scale[pages].cpu().numpy()[:, :, 0].repeat(64, 0)[:n].astype(np.float64)
    ref, tol = oa.attention(q, kc * ks[..., None], vc * vs[..., None], [0, n], [0, n], D ** -0.5, oa.CAUSAL)
    _close(many, ref, tol)
    _close(one, ref[-1:], tol[-1:])
    assert int(cache.k.count_nonzero()) == int(cache.k[pages].count_nonzero())


# ---- as a program uses them -------------------------------------------------------------------------------------------------------

def test_attention_between_the_quantized_layers():
    """LayerNorm + DAQ, qkv, attention, DAQ from its row maxima, projection with the residual: each step on what the one in front left."""
    import oracle
    import workload
    B, S, W, H = 3, 64, 384, 6
    M, D = B * S, W // H
    x = workload.activations(M, W, "attention block")
    qkv, proj = workload.layer_weights("qkv", W, 3 * W, 8, "attention block"), workload.layer_weights("proj", W, W, 8, "attention block")
    dx = _dev(x)
    ln = ql.daq_quantize_ln(dx)
    rows = ql.qgemm_w8a8(ln["q"], ln["scales"], 1, _dev(qkv["w"]), _dev(qkv["s_w"]), _dev(qkv["bias"]))
    rows = (rows * 0.01).contiguous()                     # the synthetic weights are not trained: scores of a usual size
    q, k, v = (rows[:, i * W:(i + 1) * W].unflatten(1, (H, D)) for i in range(3))
    am = torch.empty(M, dtype=torch.int32, device="cuda")
    o = ql.attention_f16(q, k, v, batch=B, row_absmax=am)
    codes, scales = ql.daq_quantize_rowmax(o.view(M, W), 1, am)
    y = ql.qgemm_w8a8(codes, scales, 1, _dev(proj["w"]), _dev(proj["s_w"]), _dev(proj["bias"]))
    torch.cuda.synchronize()
    cu = [i * S for i in range(B + 1)]
    ref, tol = oa.attention(*(t.cpu().numpy() for t in (q, k, v)), cu, cu, D ** -0.5)
    _close(o, ref, tol)
    c2, s2 = ql.daq_quantize(o.view(M, W), 1)
    assert torch.equal(codes, c2) and torch.equal(scales, s2), "codes from the row maxima"
    want = oracle.qlinear_w8a8(o.view(M, W).cpu().numpy(), 1, proj["w"], proj["s_w"], proj["bias"], nthreads=4)["y"]
    got, want = y.cpu().numpy().astype(np.float64), want.astype(np.float64)
    assert np.all(np.abs(got - want) <= np.maximum(1e-3 * np.abs(want), 2.0 ** -24))


def test_prompt_then_tokens():
    """A prompt enters the cache and attends over the values it holds; then single tokens, three at a time in one sequence, over the cache."""
    g = _rng(50)
    Hq, Hkv, D = 8, 2, 64
    c = _Cached(g, 2, 256, Hkv, D, 64, 16)
    rot = _table(256, D)
    lens = np.array([100, 37], np.int32)
    cu = _cu(lens)
    T = int(lens.sum())
    rows = _f16(g, T, (Hq + 2 * Hkv) * D)
    d = _dev(rows)
    dq, dk, dv = d[:, :Hq * D].unflatten(1, (Hq, D)), d[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D)), d[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
    k_val, v_val = (torch.empty((T, Hkv, D), dtype=torch.float16, device="cuda") for _ in range(2))
    q_rot = ql.daq_kv_append(c.dev, dk, dv, c.table, _dev(lens), cu=_dev(cu), q=dq, rot=_dev(rot), k_out=k_val, v_out=v_val)
    c.ref.append(rows[:, Hq * D:(Hq + Hkv) * D].reshape(T, Hkv, D), rows[:, (Hq + Hkv) * D:].reshape(T, Hkv, D), cu, lens, None, rot)
    c.same()
    dense = ql.attention_f16(q_rot, k_val, v_val, cu_q=_dev(cu), cu_k=_dev(cu), mask=ql.MASK_CAUSAL)
    paged = ql.attention_kv8(q_rot, c.dev, c.table, _dev(lens), cu_q=_dev(cu))
    torch.cuda.synchronize()
    ref, tol = oa.attention(q_rot.cpu().numpy(), k_val.cpu().numpy(), v_val.cpu().numpy(), cu, cu, D ** -0.5, oa.CAUSAL)
    _close(dense, ref, tol)
    ref, tol = oa.attention_cached(q_rot.cpu().numpy(), c.ref, cu, lens, D ** -0.5)
    _close(paged, ref, tol)
    for new in ([1, 1], [3, 1], [1, 0], [1, 1]):
        lens = lens + np.array(new, np.int32)
        q = _append(g, c, lens, new, Hq, rot)
        o = ql.attention_kv8(q, c.dev, c.table, _dev(lens), cu_q=_dev(_cu(new)))
        torch.cuda.synchronize()
        ref, tol = oa.attention_cached(q.cpu().numpy(), c.ref, _cu(new), lens, D ** -0.5)
        _close(o, ref, tol, str(new))


def test_captured_step_follows_its_lengths():
    """A generation step in a graph: replayed after the lengths and rows in its buffers changed, with eager work between; a second graph shares the workspace."""
    g = _rng(51)
    B, Hq, Hkv, D = 3, 8, 2, 128
    c = _Cached(g, B, 512, Hkv, D, 64, 64)
    rot = _dev(_table(512, D))
    lens = _dev(np.array([400, 60, 129], np.int32))
    rows = torch.empty((B, (Hq + 2 * Hkv) * D), dtype=torch.float16, device="cuda")
    q, k, v = rows[:, :Hq * D].unflatten(1, (Hq, D)), rows[:, Hq * D:(Hq + Hkv) * D].unflatten(1, (Hkv, D)), rows[:, (Hq + Hkv) * D:].unflatten(1, (Hkv, D))
    q_rot, o, o2 = (torch.empty((B, Hq, D), dtype=torch.float16, device="cuda") for _ in range(3))
    am = torch.empty(B, dtype=torch.int32, device="cuda")
    ws = ql.workspace(max(ql.attention_kv8_workspace_bytes(B, B, Hq, Hkv, D), ql.attention_f16_workspace_bytes(B, 512, 1, Hq, Hkv, D)))
    keys = _dev(_f16(g, 512, 2 * Hkv, D))

    def step():
        ql.daq_kv_append(c.dev, k, v, c.table, lens, q=q, rot=rot, q_out=q_rot)
        ql.attention_kv8(q_rot, c.dev, c.table, lens, o=o, row_absmax=am, ws=ws)

    def other():
        ql.attention_f16(q_rot, keys[:, :Hkv], keys[:, Hkv:], batch=1, o=o2, ws=ws)

    rows.copy_(_dev(_f16(g, *rows.shape)))
    step(), other()
    torch.cuda.synchronize()
    graphs = []
    for fn in (step, other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fn()
        graphs.append(graph)
    for turn in range(4):
        rows.copy_(_dev(_f16(g, *rows.shape, size=1.0 + turn)))
        lens.add_(1)
        saved = [t.clone() for t in (c.dev.k, c.dev.v, c.dev.k_scale, c.dev.v_scale)]
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (c.dev.k, c.dev.v, c.dev.k_scale, c.dev.v_scale, q_rot, o, am, o2)]
        for t, s in zip((c.dev.k, c.dev.v, c.dev.k_scale, c.dev.v_scale), saved):
            t.copy_(s)
        for t in (q_rot, o, o2):
            t.fill_(9.0)
        step(), other()
        torch.cuda.synchronize()
        for name, a, b in zip(("k", "v", "k_scale", "v_scale", "q", "o", "absmax", "o2"), got, (c.dev.k, c.dev.v, c.dev.k_scale, c.dev.v_scale, q_rot, o, am, o2)):
            assert torch.equal(a, b), "%s differs in replay %d" % (name, turn)


def test_results_do_not_depend_on_the_run():
    """The same call twice, and on another stream beside other work: the same bits."""
    g = _rng(52)
    q, k, v = (_dev(_f16(g, 700, 4, 72)) for _ in range(3))
    c = _Cached(g, 2, 1500, 2, 64, 64, 16)
    lens, t = _dev(np.array([1500, 700], np.int32)), _dev(_f16(g, 2, 8, 64))
    first = ql.attention_f16(q, k, v, mask=ql.MASK_CAUSAL), ql.attention_kv8(t, c.dev, c.table, lens)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        again = ql.attention_f16(q, k, v, mask=ql.MASK_CAUSAL, stream=side), ql.attention_kv8(t, c.dev, c.table, lens, stream=side.cuda_stream)
        here = ql.attention_f16(q, k, v, mask=ql.MASK_CAUSAL), ql.attention_kv8(t, c.dev, c.table, lens)
        torch.cuda.synchronize()
        for a, b, d in zip(first, again, here):
            assert torch.equal(a, b) and torch.equal(a, d)


def test_refusals_with_tensors():
    x = torch.zeros((8, 2, 64), dtype=torch.float16, device="cuda")
    odd = torch.zeros((8, 2, 68), dtype=torch.float16, device="cuda")[:, :, :64]
    with pytest.raises(ql.QlError):
        ql.attention_f16(odd, x, x)                       # heads 68 elements apart
    with pytest.raises(ql.QlError):
        ql.attention_f16(x, x, x, batch=3)                # 8 rows are no three equal sequences
    with pytest.raises(ql.QlError):
        ql.attention_f16(x, x, x, mask=ql.MASK_PREFIX)    # no prefix lengths
    with pytest.raises(TypeError):
        ql.attention_f16(x.float(), x, x)
    with pytest.raises((TypeError, ValueError)):
        ql.attention_f16(x.transpose(1, 2), x, x)         # 64 heads of 2, not next to each other
    with pytest.raises(ValueError):
        ql.attention_f16(x, x, x[:4])
    with pytest.raises(TypeError):
        ql.attention_f16(x, x, x, cu_q=torch.zeros(2, dtype=torch.int64, device="cuda"))
    cache = ql.KvCache8.empty(2, 2, 64)
    table, lens = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        ql.daq_kv_append(cache, x, x[:4], table, lens)
    with pytest.raises(ValueError):
        ql.attention_kv8(x[:, :, :32], cache, table, lens)
    with pytest.raises(ql.QlError):
        ql.daq_kv_append(cache, x, x, table, lens, rot=torch.zeros((4, 12, 2), device="cuda"))   # 24 turned channels


class _Elsewhere(torch.Tensor):
    """A tensor that says it is on another device."""

    def get_device(self):
        return torch.cuda.current_device() + 1


def test_tensors_of_another_device_are_refused():
    x = torch.zeros((8, 2, 64), dtype=torch.float16, device="cuda")
    ints, many = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    table, lens, slopes = torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(2, device="cuda")
    cache = ql.KvCache8.empty(2, 2, 64)
    there = lambda t: t.as_subclass(_Elsewhere)
    ws = ql.workspace(1 << 20)
    dense = dict(q=x, k=x, v=x, cu_q=ints, cu_k=ints, prefix=lens, slopes=slopes, o=torch.zeros_like(x), row_absmax=many, ws=ws)
    cached = dict(q=x, cache=cache, page_table=table, len_k=lens, cu_q=ints, prefix=lens, slopes=slopes, o=torch.zeros_like(x), row_absmax=many,
                  ws=ql.workspace(ql.attention_kv8_workspace_bytes(8, 1, 2, 2, 64)))
    append = dict(cache=cache, k=x, v=x, page_table=table, len_k=lens, cu=ints, q=x, rot=torch.zeros((4, 16, 2), device="cuda"), pos=many,
                  q_out=torch.zeros_like(x), k_out=torch.zeros_like(x), v_out=torch.zeros_like(x))
    for call, args in ((ql.attention_f16, dense), (ql.attention_kv8, cached), (ql.daq_kv_append, append)):
        call(**args)
        for name, t in args.items():
            moved = ql.KvCache8(there(cache.k), cache.v, cache.k_scale, cache.v_scale) if t is cache else there(t)
            with pytest.raises(ValueError, match="current device"):
                call(**{**args, name: moved})
    torch.cuda.synchronize()


# ---- values that the mask hides, long tails, scores of any size -----------------------------------------------------------------------

@pytest.mark.parametrize("mask", [1, 2])
@pytest.mark.parametrize("S", [1, 16, 32])
@pytest.mark.parametrize("nq, D", [([4, 2, 3, 1], 128), ([9, 5], 256), ([64], 64), ([70, 33], 128), ([64, 90], 40)])
def test_scales_of_hidden_tokens_do_not_count(nq, D, S, mask):
    """The first rows of a prompt see tokens of small value scale; those behind them in the same 64 have scales up to 2^20 times as large, which
    must not take the visible weights' bits.  Few rows (the first two) and many."""
    g = _rng(60, len(nq), D, S, mask)
    c = _Cached(g, len(nq), 128, 2, D, 64, S)
    jump = 20.0 * np.minimum(np.arange(64 // S) / (8 if S == 1 else 1), 1.0) - 8
    c.ref.vs *= np.tile(2.0 ** jump, c.ref.page // 64).astype(np.float32)
    c.dev.v_scale.copy_(torch.from_numpy(c.ref.vs))
    few = sum(nq) < 30                                    # their run of rows begins in front of the jump and ends behind it
    nk = [n if S == 1 or not few else S + n // 2 for n in nq]
    _cached((60, 1, len(nq), D, S, mask), nq, nk, 2, 2, D, 64, S, mask, cache=c)


@pytest.mark.parametrize("kernel", ["dense", "dense_cut", "chunks", "chunks_fine", "tokens"])
@pytest.mark.parametrize("size, scale", [(64.0, 1.0), (2000.0, 0.125), (30000.0, 0.125), (30000.0, -1.0)])
def test_scores_far_from_zero(kernel, size, scale):
    """Scores up to 2^37 in fp32, where a step of theirs is thousands: the result is still a mean of the values, each of them between 1 and 2.  A mean may
    pass them by the rounding of its binary16 weights and of its own, 2 x 2^-11 of 2; its place between them is the fp32 scores' rounding."""
    g = _rng(61, int(size))
    D, n, H = 64, 300, 2
    rows = 1 if kernel == "tokens" else 20 if kernel == "dense_cut" else 300
    q = _f16(g, rows, H, D, size=0.0) + np.float16(size)
    k = (size * g.uniform(0.5, 1.0, (n, H, D))).astype(np.float16)
    v = g.uniform(1.0, 2.0, (n, H, D)).astype(np.float16)
    if kernel.startswith("dense"):
        o = ql.attention_f16(_dev(q), _dev(np.concatenate([k] * (8 if kernel == "dense_cut" else 1))), _dev(np.concatenate([v] * (8 if kernel == "dense_cut" else 1))), scale=scale)
    else:
        S = 16 if kernel == "chunks_fine" else 64
        cache = ql.KvCache8.empty(6, H, D, page=64, scale_tokens=S)
        table, lens = _dev(np.array([[4, 0, 2, 5, 1]], np.int32)), _dev(np.array([n], np.int32))
        ql.daq_kv_append(cache, _dev(k), _dev(v), table, lens)
        o = ql.attention_kv8(_dev(q), cache, table, lens, mask=ql.MASK_NONE, scale=scale)
    torch.cuda.synchronize()
    o = o.float().cpu().numpy()
    edge = 2.0 * 2.0 * 2.0 ** -11 + (0.0 if kernel.startswith("dense") else 0.5 * 2.0 / 127 * (1 + 2.0 ** -7))   # a code is off by half a step
    assert np.isfinite(o).all() and o.min() >= 1.0 - edge and o.max() <= 2.0 + edge, (o.min(), o.max())


@pytest.mark.parametrize("S", [1, 16, 64])
@pytest.mark.parametrize("nq, nk", [([1, 1], [300, 170]), ([150, 90], [300, 170])])
def test_value_scales_next_to_zero(nq, nk, S):
    """Scales whose reciprocal passes fp32, in whole sequences and in front of ordinary ones."""
    g = _rng(62, sum(nq), S)
    c = _Cached(g, 2, 320, 2, 64, 64, S)
    for b, pages in ((0, 5), (1, 1)):
        for i in range(pages):
            c.ref.vs[c.ref.table[b, i]] = np.float32((1e-39, 1e-42, 0.0, 1e-30, 1e-45)[i])
    c.dev.v_scale.copy_(torch.from_numpy(c.ref.vs))
    _cached((62, 1, sum(nq), S), nq, nk, 4, 2, 64, 64, S, cache=c)


def _sink_and_tail(g, n, sinks, D, gap):
    """Keys whose scores lie `gap` nats below those of a few, n of them, with values of the other sign: together they move the result by n e^-gap / sinks."""
    k, v = np.zeros((n, 1, D), np.int8), g.integers(64, 128, (n, 1, D)).astype(np.int8)
    for j in sinks:
        k[j], v[j] = 127, -127
    return k, v, np.float32(gap / (D * 127)), np.float32(1.0 / 127)


def test_long_tails_below_a_sink_dense():
    """One key far above 131070 others: their weights are tiny, their sum is not.  256 heads read the same keys, so that no part of the keys is a
    workgroup's of its own and every row has the one maximum."""
    g = _rng(63)
    n, D, H, gap = 131071, 64, 256, 17.4
    k, v, ks, vs = _sink_and_tail(g, n, [70000], D, gap)
    k = (k.astype(np.float32) * ks).astype(np.float16)
    v = (v.astype(np.float32) * vs).astype(np.float16)
    q = np.ones((1, 1, D), np.float16)
    ref, tol = oa.attention(q, k, v, [0, 1], [0, n], 1.0)
    o = ql.attention_f16(_dev(q).expand(1, H, D).contiguous(), _dev(k).expand(n, H, D), _dev(v).expand(n, H, D), scale=1.0)
    torch.cuda.synchronize()
    _close(o, np.repeat(ref, H, 1), np.repeat(tol, H, 1))


@pytest.mark.parametrize("rows, H, D, n, S", [(1, 2048, 8, 524288, 64), (1, 2048, 8, 524288, 16), (512, 128, 64, 131072, 64), (512, 128, 64, 131072, 1)])
def test_long_tails_below_a_sink_cached(rows, H, D, n, S):
    """The same over the cache, by 16 rows (each of a workgroup's wavefronts has a sink of its own in its first group) and by 256.  The tail is one
    page again and again."""
    g = _rng(64, rows, S)
    gap = 17.4
    few = rows == 1
    front = 256 if few else 64
    sinks = [3, 70, 140, 255] if few else [17]
    fk, fv, ks, vs = _sink_and_tail(g, front, sinks, D, gap)
    tk, tv, _, _ = _sink_and_tail(g, 64, [], D, gap)
    pages = front // 64 + 1
    ck, cv = np.concatenate((fk, tk)), np.concatenate((fv, tv))                  # [pages * 64, 1, D]
    kc = np.broadcast_to(ck.reshape(pages, 64, D)[:, None], (pages, H, 64, D))
    order = np.argsort([oa.slot(t) for t in range(64)])                           # byte -> token
    vc = np.broadcast_to(cv.reshape(pages, 64, D)[:, order].transpose(0, 2, 1)[:, None, None], (pages, H, 1, D, 64))
    scales = np.ones((pages, H, 64 // S), np.float32)
    cache = ql.KvCache8(_dev(kc), _dev(vc), _dev(scales * ks), _dev(scales * vs))
    table = np.full((1, n // 64), pages - 1, np.int32)
    table[0, :pages - 1] = np.arange(pages - 1)
    q = np.ones((1, 1, D), np.float16)
    o = ql.attention_kv8(_dev(np.broadcast_to(q, (rows, H, D))), cache, _dev(table), _dev(np.array([n], np.int32)), mask=ql.MASK_NONE, scale=1.0)
    k, v = (np.concatenate((f, np.tile(t, ((n - front) // 64, 1, 1)))) for f, t in ((fk, tk), (fv, tv)))
    ref, tol = oa.attention(q, k * np.float64(ks), v * np.float64(vs), [0, 1], [0, n], 1.0)
    torch.cuda.synchronize()
    _close(o, np.broadcast_to(ref, (rows, H, D)), np.broadcast_to(tol, (rows, H, D)))


def _making_its_tensors(name):
    """A call that makes its output and workspace itself, always with the same result."""
    g = _rng(65)
    q, k, v = (_dev(_f16(g, 256, 4, 64)) for _ in range(3))
    c = _Cached(g, 1, 256, 4, 64, 64, 64)
    lens = _dev(np.array([256], np.int32))
    calls = {"attention_f16": lambda **kw: ql.attention_f16(q, k, v, **kw), "attention_kv8": lambda **kw: ql.attention_kv8(q, c.dev, c.table, lens, **kw),
             "daq_kv_append": lambda **kw: ql.daq_kv_append(c.dev, k, v, c.table, lens, q=q, **kw)}
    return calls[name]


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("name", ["attention_f16", "attention_kv8", "daq_kv_append"])
def test_tensors_made_for_another_stream(name, handle):
    """Memory freed on the current stream, where a fill still waits, is not what a call on another stream writes to; nor does a later call there write to what
    the current stream still reads of an earlier result."""
    side = torch.cuda.Stream()
    call = _making_its_tensors(name)
    want = call()
    torch.cuda.synchronize()
    there = dict(stream=side.cuda_stream if handle else side)
    torch.cuda._sleep(20_000_000)
    for _ in range(4):
        junk = torch.empty_like(want)
        junk.fill_(7.0)
        del junk
    got = call(**there)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(20_000_000)
    kept = got.clone()
    del got
    for _ in range(3):
        with torch.cuda.stream(side):
            torch.empty_like(want).fill_(9.0)
        call(**there)
    torch.cuda.synchronize()
    assert torch.equal(kept, want)


def test_one_workspace_for_all_smaller_calls():
    """A program takes its workspace once, for the most rows that it will have."""
    g = _rng(66)
    Hq, Hkv, D, n = 16, 2, 64, 4096
    q, k, v = _dev(_f16(g, n, Hq, D)), _dev(_f16(g, n, Hkv, D)), _dev(_f16(g, n, Hkv, D))
    c = _Cached(g, 1, n, Hkv, D, 64, 64)
    lens = _dev(np.array([n], np.int32))
    dense, cached = ql.workspace(ql.attention_f16_workspace_bytes(n, n, 1, Hq, Hkv, D)), ql.workspace(ql.attention_kv8_workspace_bytes(n, 1, Hq, Hkv, D))
    for T in (1, 3, 64, 256, 512, 1024, 2048, 4096):
        a = ql.attention_f16(q[:T], k, v, ws=dense), ql.attention_kv8(q[:T], c.dev, c.table, lens, ws=cached)
        b = ql.attention_f16(q[:T], k, v), ql.attention_kv8(q[:T], c.dev, c.table, lens)
        torch.cuda.synchronize()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
