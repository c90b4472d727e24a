"""Refusals of the attention and cache calls (made before the first HIP call, so without a GPU), the cache's storage order and the oracle's pins."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2511_11446_amd as ql
from oracle import attention as oa

A = 0x10000          # never dereferenced: every call below has to fail its checks first
BIG = 1 << 40


def _attn(**kw):
    a = dict(T_q=64, B=2, Hq=4, Hkv=2, D=64, mask=0, scale=0.125, cap=0.0, reserved=0, prefix=None, slopes=None, cu_q=None, q=A, q_row=256, q_head=64,
             o=A, o_row=256, o_head=64, row_absmax=None)
    a.update(kw)
    return ql.ql_attention(**a)


def _f16(a, k=A, k_row=128, k_head=64, v=A, v_row=128, v_head=64, T_k=64, cu_k=None, ws=A, nbytes=BIG):
    return ql.lib().attention_f16(ctypes.byref(a) if a is not None else None, k, k_row, k_head, v, v_row, v_head, T_k, cu_k, ws, nbytes, None)


@pytest.mark.parametrize("kw, status", [
    (dict(q=None), 1), (dict(o=None), 1), (dict(mask=2), 1),                                             # a pointer is missing
    (dict(mask=3), 4), (dict(mask=-1), 4), (dict(reserved=1), 4), (dict(scale=float("nan")), 4), (dict(scale=float("inf")), 4),
    (dict(cap=-1.0), 4), (dict(cap=float("nan")), 4), (dict(cap=float("inf")), 4), (dict(cap=2.0 ** -10 * (1 - 2.0 ** -20)), 4), (dict(cap=1025.0), 4),
    (dict(T_q=0), 2), (dict(B=0), 2), (dict(Hq=0), 2), (dict(Hkv=0), 2), (dict(Hq=3), 2), (dict(D=0), 2), (dict(D=60), 2), (dict(D=264), 2),
    (dict(T_q=63), 2), (dict(T_q=1 << 31), 2), (dict(T_q=1 << 30), 2), (dict(B=1 << 19, cu_q=A), 2),     # unequal lengths, too many rows or sequences
    (dict(q_row=(1 << 24) + 8), 2),
    (dict(q_row=252), 2), (dict(q_head=-64), 2), (dict(o_row=0), 2), (dict(o_head=32), 2), (dict(o_row=192), 2),   # outputs that overlap
    (dict(q=A + 8), 3), (dict(o=A + 2), 3), (dict(slopes=A + 2), 3), (dict(cu_q=A + 1), 3), (dict(row_absmax=A + 3), 3), (dict(mask=2, prefix=A + 2), 3),
])
def test_attention_argument_checks(kw, status):
    assert _f16(_attn(**kw)) == status
    c = _cache()
    assert ql.lib().attention_kv8(ctypes.byref(_attn(**kw)), ctypes.byref(c), A, BIG, None) == status


@pytest.mark.parametrize("kw, status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(T_k=0), 2), (dict(T_k=63), 2), (dict(T_k=1 << 31), 2), (dict(k_row=4), 2), (dict(v_head=-8), 2),
    (dict(k=A + 4), 3), (dict(v=A + 8), 3), (dict(cu_k=A + 2), 3)])
def test_attention_f16_key_checks(kw, status):
    assert _f16(_attn(), **kw) == status


def test_attention_workspace_checks():
    assert _f16(None) == 1
    need = ql.attention_f16_workspace_bytes(64, 64, 2, 4, 2, 64)
    if need:
        assert _f16(_attn(), ws=None) == 5 and _f16(_attn(), nbytes=need - 1) == 5 and _f16(_attn(), ws=A + 16) == 3
    need = ql.attention_kv8_workspace_bytes(64, 2, 4, 2, 64)
    L, a, c = ql.lib(), _attn(), _cache()
    if need:
        assert L.attention_kv8(ctypes.byref(a), ctypes.byref(c), None, BIG, None) == 5
        assert L.attention_kv8(ctypes.byref(a), ctypes.byref(c), A, need - 1, None) == 5
        assert L.attention_kv8(ctypes.byref(a), ctypes.byref(c), A + 16, BIG, None) == 3
    assert L.attention_kv8(None, ctypes.byref(c), A, BIG, None) == 1
    assert L.attention_kv8(ctypes.byref(a), None, A, BIG, None) == 1
    for fn, arg in ((ql.attention_f16_workspace_bytes, (0, 1, 1, 1, 1, 64)), (ql.attention_kv8_workspace_bytes, (1, 0, 1, 1, 64))):
        assert fn(*arg) == 0                                        # sizes that the call refuses


def _cache(**kw):
    c = dict(k=A, v=A, k_scale=A, v_scale=A, num_pages=8, page=64, scale_tokens=64, Hkv=2, D=64, page_table=A, len_k=A, B=2, max_pages=4)
    c.update(kw)
    return ql.ql_kv_cache(**c)


CACHE_REFUSALS = [
    (dict(k=None), 1), (dict(v=None), 1), (dict(k_scale=None), 1), (dict(v_scale=None), 1), (dict(page_table=None), 1), (dict(len_k=None), 1),
    (dict(scale_tokens=0), 4), (dict(scale_tokens=8), 4), (dict(scale_tokens=128), 4),
    (dict(page=32), 2), (dict(page=96), 2), (dict(page=0), 2), (dict(num_pages=0), 2), (dict(num_pages=1 << 31), 2), (dict(max_pages=0), 2),
    (dict(max_pages=1 << 26), 2), (dict(B=0), 2), (dict(Hkv=0), 2), (dict(D=12), 2), (dict(D=320), 2),
    (dict(k=A + 8), 3), (dict(v=A + 4), 3), (dict(k_scale=A + 2), 3), (dict(v_scale=A + 1), 3), (dict(page_table=A + 2), 3), (dict(len_k=A + 2), 3)]


def _new(**kw):
    n = dict(T=64, Hq=4, rot_pairs=0, cu=None, q=A, k=A, v=A, q_row=256, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, rot=A, rot_rows=100,
             rot_dim=64, reserved=0, pos=None, q_out=A, k_out=None, v_out=None)
    n.update(kw)
    return ql.ql_kv_new(**n)


@pytest.mark.parametrize("kw, status", CACHE_REFUSALS)
def test_cache_argument_checks(kw, status):
    L, c = ql.lib(), _cache(**kw)
    n = _new()
    assert L.daq_kv_append(ctypes.byref(c), ctypes.byref(n), None) == status
    a = _attn()
    assert L.attention_kv8(ctypes.byref(a), ctypes.byref(c), A, BIG, None) == status


@pytest.mark.parametrize("kw, status", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(q=None), 1), (dict(reserved=1), 4), (dict(rot_pairs=2), 4), (dict(T=0), 2), (dict(T=63), 2),
    (dict(T=1 << 32), 2), (dict(Hq=0), 2), (dict(Hq=3), 2), (dict(k_row=12), 2), (dict(v_row=-8), 2), (dict(q_head=4), 2), (dict(rot_dim=8), 2),
    (dict(rot_dim=72), 2), (dict(rot_dim=80), 2), (dict(rot_rows=0), 2), (dict(k=A + 2), 3), (dict(v=A + 8), 3), (dict(q=A + 8), 3), (dict(rot=A + 4), 3),
    (dict(q_out=A + 8), 3), (dict(k_out=A + 8), 3), (dict(v_out=A + 8), 3), (dict(cu=A + 2), 3), (dict(pos=A + 2), 3)])
def test_append_argument_checks(kw, status):
    L, c, n = ql.lib(), _cache(), _new(**kw)
    assert L.daq_kv_append(ctypes.byref(c), ctypes.byref(n), None) == status
    assert L.daq_kv_append(ctypes.byref(c), None, None) == 1


def test_attention_and_cache_must_fit():
    L, c = ql.lib(), _cache()
    for kw in (dict(B=4), dict(Hkv=4), dict(D=128, q_row=512, q_head=128, o_row=512, o_head=128)):
        a = _attn(**kw)
        assert L.attention_kv8(ctypes.byref(a), ctypes.byref(c), A, BIG, None) == 2


def test_binding_refuses_tensors_of_the_wrong_kind():
    x = torch.zeros((4, 2, 64), dtype=torch.float16)                  # not on a GPU
    with pytest.raises(TypeError):
        ql.attention_f16(x, x, x)
    with pytest.raises(TypeError):
        ql.KvCache8(torch.zeros((1, 1, 64, 64), dtype=torch.int8), None, None, None)


def test_storage_order_of_value_codes():
    """A permutation of a group's tokens; the four that one lane reads of a 16-token tile lie together."""
    s = [oa.slot(t) for t in range(64)]
    assert sorted(s) == list(range(64))
    assert s[:4] == [0, 1, 2, 3] and s[4:8] == [16, 17, 18, 19] and s[16:20] == [4, 5, 6, 7] and s[63] == 63


def test_oracle_attention_against_torch():
    g = np.random.default_rng(7)
    q, k, v = (g.standard_normal((9, 4, 16)) for _ in range(3))
    for mask in (oa.NONE, oa.CAUSAL):
        o, _ = oa.attention(q, k[:, :2], v[:, :2], [0, 9], [0, 9], 0.3, mask)
        t = [torch.from_numpy(x).transpose(0, 1) for x in (q, np.repeat(k[:, :2], 2, 1), np.repeat(v[:, :2], 2, 1))]
        ref = torch.nn.functional.scaled_dot_product_attention(*t, is_causal=mask == oa.CAUSAL, scale=0.3).transpose(0, 1).numpy()
        assert np.abs(o - ref).max() < 1e-12


def test_oracle_attention_hand_worked():
    """Two keys, weights 1 : 3; the cap and the bias each turn the scores into the same ones; a row that sees nothing is zero."""
    q, v = np.ones((1, 1, 1)), np.array([[[4.0]], [[8.0]]])
    k = np.array([[[0.0]], [[np.log(3.0)]]])
    assert abs(oa.attention(q, k, v, [0, 1], [0, 2], 1.0)[0][0, 0, 0] - 7.0) < 1e-12
    assert abs(oa.attention(q, np.zeros_like(k), v, [0, 1], [0, 2], 1.0, slopes=[np.log(3.0)])[0][0, 0, 0] - 7.0) < 1e-12
    capped = np.array([[[0.0]], [[2.0 * np.arctanh(np.log(3.0) / 2.0)]]])
    assert abs(oa.attention(q, capped, v, [0, 1], [0, 2], 1.0, cap=2.0)[0][0, 0, 0] - 7.0) < 1e-12
    o, _ = oa.attention(np.ones((2, 1, 1)), k[1:], v[1:], [0, 2], [0, 1], 1.0, mask=oa.CAUSAL)
    assert o[0, 0, 0] == 0.0 and o[1, 0, 0] == 8.0


def test_oracle_append_hand_worked():
    """Scale 1 from a maximum of 127; a second token of 254 doubles it, and the codes in front are halved (ties to even)."""
    D = 8
    c = oa.Cache(np.zeros((1, 1, 64, D), np.int8), np.zeros((1, 1, 1, D, 64), np.int8), np.zeros((1, 1, 1), np.float32), np.zeros((1, 1, 1), np.float32),
                 np.zeros((1, 1), np.int32))
    x = np.array([127, 1, 2, 3, 5, -1, -3, 0], np.float16).reshape(1, 1, D)
    c.append(x, x, [0, 1], [1])
    assert c.ks[0, 0, 0] == 1.0 and list(c.kc[0, 0, 0]) == [127, 1, 2, 3, 5, -1, -3, 0] and list(c.vc[0, 0, 0, :, 0]) == [127, 1, 2, 3, 5, -1, -3, 0]
    y = np.array([254, 0, 0, 0, 0, 0, 0, 2], np.float16).reshape(1, 1, D)
    out = c.append(y, y, [0, 1], [2])
    assert c.ks[0, 0, 0] == 2.0 and list(c.kc[0, 0, 0]) == [64, 0, 1, 2, 2, 0, -2, 0] and list(c.kc[0, 0, 1]) == [127, 0, 0, 0, 0, 0, 0, 1]
    assert list(out["k_out"][0, 0]) == [254, 0, 0, 0, 0, 0, 0, 2]


def test_oracle_rotation_is_a_rotation():
    g = np.random.default_rng(3)
    x = g.standard_normal((2, 32)).astype(np.float16)
    a = g.uniform(0, 6, 8)
    row = np.stack((np.cos(a), np.sin(a)), -1).astype(np.float32)
    for pairs in (False, True):
        y = oa.rotate(x, row, pairs).astype(np.float64)
        i = 2 * np.arange(8) if pairs else np.arange(8)
        j = i + 1 if pairs else i + 8
        z = (x[:, i].astype(np.float64) + 1j * x[:, j]) * np.exp(1j * a)
        assert np.abs(y[:, i] - z.real).max() < 4e-3 and np.abs(y[:, j] - z.imag).max() < 4e-3     # |z| < 4: half a binary16 step is 2^-10
        assert np.array_equal(y[:, 16:], x[:, 16:].astype(np.float64))


@pytest.mark.parametrize("Hq, Hkv, D", [(1, 1, 64), (16, 2, 128), (32, 8, 256), (40, 40, 72), (6, 6, 8)])
def test_workspace_for_the_largest_call_is_enough_for_smaller_ones(Hq, Hkv, D):
    """Fewer rows may be cut into more parts: the size is that of the worst call up to the one that is asked for."""
    rows = [1, 2, 16, 17, 64, 128, 200, 256, 300, 512, 777, 1024, 2048, 4096, 5000, 8192, 65536]
    keys = [1, 64, 255, 512, 1024, 4095, 8192, 131071]
    for B in (1, 2, 7, 64, 300):
        for T_k in keys:
            sizes = [ql.attention_f16_workspace_bytes(t, T_k, B, Hq, Hkv, D) for t in rows]
            assert sizes == sorted(sizes), (B, T_k)
        for t in rows:
            sizes = [ql.attention_f16_workspace_bytes(t, T_k, B, Hq, Hkv, D) for T_k in keys]
            assert sizes == sorted(sizes), (B, t)
        sizes = [ql.attention_kv8_workspace_bytes(t, B, Hq, Hkv, D) for t in rows]
        assert sizes == sorted(sizes), B
    for t in rows:
        for fn in (lambda B: ql.attention_f16_workspace_bytes(t, 8192, B, Hq, Hkv, D), lambda B: ql.attention_kv8_workspace_bytes(t, B, Hq, Hkv, D)):
            sizes = [fn(B) for B in (1, 2, 7, 64, 300)]
            assert sizes == sorted(sizes), t
