"""Refusals of the 8-bit floating point, routing and experts' calls (made before the first HIP call, so without a GPU), the structures that the binding packs, the memory
of what it makes, and the oracle's pins."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2511_11446_amd as ql
from oracle import f8 as of
from test_binding_streams_cpu import CURRENT, _OnTheOther, _Stream, _t, made  # noqa: F401

A = 0x10000          # never dereferenced: every call below has to fail its checks first
BIG = 1 << 40
F8 = torch.float8_e4m3fn


def _fusion(**kw):
    f = dict(act=0, reserved=0, residual=None, gate=None, gate_rows=1, row_absmax=None)
    f.update(kw)
    return ctypes.byref(ql.ql_fusion(**f))


@pytest.mark.parametrize("kw, status", [
    (dict(x=None), 1), (dict(q=None), 1), (dict(s=None), 1), (dict(glu=2), 4), (dict(glu=-1), 4), (dict(M=0), 2), (dict(K=0), 2), (dict(K=8), 2), (dict(K=136), 2),
    (dict(M=1 << 24), 2), (dict(M=1 << 23, K=128, glu=1), 2), (dict(x=A + 8), 3), (dict(q=A + 8), 3), (dict(s=A + 2), 3)])
def test_quantizer_checks(kw, status):
    a = dict(x=A, M=4, K=128, glu=0, q=A, s=A)
    a.update(kw)
    assert ql.lib().daq_quantize_f8(a["x"], a["M"], a["K"], a["glu"], a["q"], a["s"], None) == status


LAYER = [(dict(w=None), 1), (dict(sw=None), 1), (dict(y=None), 1), (dict(M=0), 2), (dict(N=0), 2), (dict(K=120), 2), (dict(K=-16), 2), (dict(M=1 << 24), 2), (dict(N=1 << 24), 2),
         (dict(M=1 << 16, N=1 << 15), 2), (dict(w=A + 8), 3), (dict(y=A + 8), 3), (dict(sw=A + 2), 3), (dict(bias=A + 1), 3),
         (dict(f=dict(act=2)), 4), (dict(f=dict(act=-1)), 4), (dict(f=dict(reserved=1)), 4), (dict(f=dict(row_absmax=A)), 4), (dict(f=dict(gate=A, gate_rows=0)), 2),
         (dict(f=dict(gate=A, gate_rows=3)), 2), (dict(f=dict(gate=A + 1)), 3), (dict(f=dict(residual=A + 1)), 3)]


@pytest.mark.parametrize("kw, status", LAYER + [(dict(q=None), 1), (dict(s=None), 1), (dict(q=A + 4), 3), (dict(s=A + 1), 3)])
def test_product_checks(kw, status):
    a = dict(q=A, s=A, M=4, K=128, w=A, sw=A, bias=None, N=64, f=None, y=A)
    a.update(kw)
    f = None if a["f"] is None else _fusion(**a["f"])
    assert ql.lib().qgemm_f8(a["q"], a["s"], a["M"], a["K"], a["w"], a["sw"], a["bias"], a["N"], f, a["y"], None) == status


@pytest.mark.parametrize("kw, status", LAYER + [(dict(x=None), 1), (dict(x=A + 2), 3), (dict(glu=3), 4), (dict(ws=None), 5), (dict(nbytes=512), 5), (dict(ws=A + 16), 3)])
def test_layer_checks(kw, status):
    a = dict(x=A, M=4, K=128, glu=0, w=A, sw=A, bias=None, N=64, f=None, y=A, ws=A, nbytes=BIG)
    a.update(kw)
    f = None if a["f"] is None else _fusion(**a["f"])
    assert ql.lib().qlinear_f8(a["x"], a["M"], a["K"], a["glu"], a["w"], a["sw"], a["bias"], a["N"], f, a["y"], a["ws"], a["nbytes"], None) == status
    need = ql.qlinear_f8_workspace_bytes(4, 128, 64)
    assert need >= 4 * 128 + 16 and ql.qlinear_f8_workspace_bytes(4, 120, 64) == 0 and ql.qlinear_f8_workspace_bytes(1000, 128, 64) >= need


@pytest.mark.parametrize("kw, status", [
    (dict(logits=None), 1), (dict(ids=None), 1), (dict(weights=None), 1), (dict(score=2), 4), (dict(score=-1), 4), (dict(logits_fp32=2), 4), (dict(renorm=2), 4),
    (dict(group_top=0), 4), (dict(group_top=3), 4), (dict(reserved=1), 4), (dict(scale=float("nan")), 4), (dict(scale=float("inf")), 4),
    (dict(T=0), 2), (dict(T=1 << 26), 2), (dict(E=0), 2), (dict(E=513), 2), (dict(k=0), 2), (dict(k=65), 2), (dict(E=64, k=64, groups=5), 2), (dict(groups=0), 2), (dict(groups=3), 2),
    (dict(E=512, groups=256), 2), (dict(top_groups=0), 2), (dict(top_groups=2), 2), (dict(E=4, k=5), 2), (dict(logits=A + 1), 3), (dict(logits=A + 2, logits_fp32=1), 3),
    (dict(bias=A + 2), 3), (dict(ids=A + 2), 3), (dict(weights=A + 1), 3)])
def test_routing_checks(kw, status):
    r = dict(T=4, E=64, k=4, score=0, logits_fp32=0, groups=1, top_groups=1, group_top=2, renorm=1, scale=1.0, reserved=0, logits=A, bias=None, ids=A, weights=A)
    r.update(kw)
    assert ql.lib().route_experts(ctypes.byref(ql.ql_routing(**r)), None) == status
    assert ql.lib().route_experts(None, None) == 1


@pytest.mark.parametrize("kw, status", [(dict([(n, None)]), 1) for n in ("x", "ids", "weights", "w_up", "up_scale", "w_down", "down_scale", "y")] + [
    (dict(T=0), 2), (dict(k=0), 2), (dict(k=65), 2), (dict(E=0), 2), (dict(E=513), 2), (dict(K=136), 2), (dict(I=24), 2), (dict(N=12), 2), (dict(T=(1 << 23) + 1, k=2, K=16, I=16, N=8), 2),
    (dict(T=1 << 23, K=256), 2), (dict(T=1 << 20, I=1 << 10), 2), (dict(T=1 << 20, N=1 << 10), 2), (dict(K=1 << 16, I=1 << 15), 2), (dict(N=1 << 16, I=1 << 15), 2),
    (dict(x=A + 8), 3), (dict(w_up=A + 8), 3), (dict(w_down=A + 4), 3), (dict(residual=A + 8), 3), (dict(y=A + 8), 3), (dict(ids=A + 2), 3), (dict(weights=A + 2), 3),
    (dict(up_scale=A + 1), 3), (dict(down_scale=A + 2), 3), (dict(ws=None), 5), (dict(nbytes=1000), 5), (dict(ws=A + 16), 3)])
def test_experts_checks(kw, status):
    e = dict(T=4, k=2, E=8, K=128, I=128, N=128, x=A, ids=A, weights=A, w_up=A, up_scale=A, w_down=A, down_scale=A, residual=None, y=A)
    ws, nbytes = kw.get("ws", A), kw.get("nbytes", BIG)
    e.update({n: v for n, v in kw.items() if n not in ("ws", "nbytes")})
    assert ql.lib().experts_f8(ctypes.byref(ql.ql_experts_f8(**e)), ws, nbytes, None) == status
    assert ql.lib().experts_f8(None, A, BIG, None) == 1


def test_a_workspace_is_enough_for_fewer_tokens():
    assert ql.experts_f8_workspace_bytes(4, 2, 8, 136, 128, 128) == 0
    for E in (1, 8, 512):
        sizes = [ql.experts_f8_workspace_bytes(T, 2, E, 256, 144, 136) for T in (1, 2, 3, 15, 16, 17, 63, 64, 65, 127, 128, 500, 511, 512, 513, 1024, 2000, 4096, 16384, 40000)]
        assert sizes == sorted(sizes) and sizes[0] > 0


def test_packed_structures_are_the_headers():
    r = ql.ql_routing(7, 1, 2, 3, 4, 5, 6, 7, 8, 0.5, 9, 10, 11, 12, 13)
    assert bytes(r) == ql._ROUTING.pack(7, 1, 2, 3, 4, 5, 6, 7, 8, 0.5, 9, 10, 11, 12, 13)
    e = ql.ql_experts_f8(7, 1, 2, 3, 4, 5, *range(6, 15))
    assert bytes(e) == ql._EXPERTS.pack(7, 1, 2, 3, 4, 5, *range(6, 15))


def _f8(*shape):
    return _t(*shape, dtype=torch.uint8).view(F8)


def _f32(*shape):
    return _t(*shape, dtype=torch.float32)


CALLS = {
    "daq_quantize_f8": lambda **kw: ql.daq_quantize_f8(_t(8, 256), **kw),
    "qgemm_f8": lambda **kw: ql.qgemm_f8(_f8(8, 256), _f32(8, 2), _f8(32, 256), _f32(1, 2), **kw),
    "qlinear_f8": lambda **kw: ql.qlinear_f8(_t(8, 256), _f8(32, 256), _f32(1, 2), **kw),
    "route_experts": lambda **kw: ql.route_experts(_t(8, 64), 4, **kw),
    "experts_f8": lambda **kw: ql.experts_f8(_t(8, 256), _t(8, 2, dtype=torch.int32), _f32(8, 2), _f8(4, 2, 128, 256), _f32(4, 2, 1, 2), _f8(4, 256, 128), _f32(4, 2, 1), **kw),
}


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("stream, handle", [(_Stream(0x50), 0x50), (0x50, 0x50), (0, 0), (None, 0)])
def test_memory_is_of_the_stream_that_the_call_runs_on(name, stream, handle, made):  # noqa: F811
    out = CALLS[name](stream=stream)
    assert made and all(t.memory_of.cuda_stream == handle for t in made)
    for t in out if isinstance(out, tuple) else [out]:
        assert stream is None or CURRENT in t.__dict__.get("used_on", []) or t.memory_of == CURRENT


@pytest.mark.parametrize("name", sorted(CALLS))
def test_the_stream_is_on_the_current_device(name, made):  # noqa: F811
    s = _Stream(0x50)
    s.device_index = 1
    with pytest.raises(ValueError, match="stream is on cuda:1"):
        CALLS[name](stream=s)


def _other(t):
    return t.as_subclass(_OnTheOther)


REFUSED = {
    "x elsewhere": lambda: ql.daq_quantize_f8(_other(_t(8, 256))),
    "x of another type": lambda: ql.daq_quantize_f8(_f32(8, 256)),
    "x strided": lambda: ql.daq_quantize_f8(_t(8, 512)[:, :256]),
    "x of three dimensions": lambda: ql.daq_quantize_f8(_t(2, 4, 256)),
    "x of one half": lambda: ql.daq_quantize_f8(_t(8, 257), glu=True),
    "q of other rows": lambda: ql.daq_quantize_f8(_t(8, 256), q=_f8(7, 256)),
    "scales of other blocks": lambda: ql.daq_quantize_f8(_t(8, 256), scales=_f32(8, 1)),
    "q in integers": lambda: ql.daq_quantize_f8(_t(8, 256), q=_t(8, 256, dtype=torch.int8)),
    "no scales": lambda: ql.qgemm_f8(_f8(8, 256), None, _f8(32, 256), _f32(1, 2)),
    "w of other inputs": lambda: ql.qlinear_f8(_t(8, 256), _f8(32, 128), _f32(1, 1)),
    "w elsewhere": lambda: ql.qlinear_f8(_t(8, 256), _other(_f8(32, 256)), _f32(1, 2)),
    "w_scale of other blocks": lambda: ql.qlinear_f8(_t(8, 256), _f8(32, 256), _f32(2, 2)),
    "no w_scale": lambda: ql.qlinear_f8(_t(8, 256), _f8(32, 256), None),
    "bias of other outputs": lambda: ql.qlinear_f8(_t(8, 256), _f8(32, 256), _f32(1, 2), bias=_t(31)),
    "residual of other rows": lambda: ql.qlinear_f8(_t(8, 256), _f8(32, 256), _f32(1, 2), residual=_t(7, 32)),
    "gate rows": lambda: ql.qlinear_f8(_t(8, 256), _f8(32, 256), _f32(1, 2), gate=_t(8, 32), gate_rows=3),
    "y of other rows": lambda: ql.qlinear_f8(_t(8, 256), _f8(32, 256), _f32(1, 2), y=_t(9, 32)),
    "ws elsewhere": lambda: ql.qlinear_f8(_t(8, 256), _f8(32, 256), _f32(1, 2), ws=_other(_t(4096, dtype=torch.uint8))),
    "logits of integers": lambda: ql.route_experts(_t(8, 64, dtype=torch.int32), 2),
    "bias of other experts": lambda: ql.route_experts(_t(8, 64), 2, bias=_f32(63)),
    "ids of other choices": lambda: ql.route_experts(_t(8, 64), 2, ids=_t(8, 3, dtype=torch.int32)),
    "ids of other tokens": lambda: ql.experts_f8(_t(8, 256), _t(7, 2, dtype=torch.int32), _f32(7, 2), _f8(4, 2, 128, 256), _f32(4, 2, 1, 2), _f8(4, 256, 128), _f32(4, 2, 1)),
    "weights of other choices": lambda: ql.experts_f8(_t(8, 256), _t(8, 2, dtype=torch.int32), _f32(8, 3), _f8(4, 2, 128, 256), _f32(4, 2, 1, 2), _f8(4, 256, 128), _f32(4, 2, 1)),
    "one matrix for gate and up": lambda: ql.experts_f8(_t(8, 256), _t(8, 2, dtype=torch.int32), _f32(8, 2), _f8(4, 256, 256), _f32(4, 2, 2), _f8(4, 256, 128), _f32(4, 2, 1)),
    "w_down of other experts": lambda: ql.experts_f8(_t(8, 256), _t(8, 2, dtype=torch.int32), _f32(8, 2), _f8(4, 2, 128, 256), _f32(4, 2, 1, 2), _f8(5, 256, 128), _f32(5, 2, 1)),
    "up_scale of other blocks": lambda: ql.experts_f8(_t(8, 256), _t(8, 2, dtype=torch.int32), _f32(8, 2), _f8(4, 2, 128, 256), _f32(4, 2, 2, 2), _f8(4, 256, 128), _f32(4, 2, 1)),
}


@pytest.mark.parametrize("what", sorted(REFUSED))
def test_the_binding_refuses(what, made):  # noqa: F811
    with pytest.raises((TypeError, ValueError)):
        REFUSED[what]()


# ---- the oracle -----------------------------------------------------------------------------------------------------------------

def test_oracle_codes_are_the_formats():
    """Against torch's own e4m3: every code's value, and the rounding of numbers in all of its range."""
    codes = np.arange(256, dtype=np.uint8)
    v = torch.from_numpy(codes).view(F8).float().numpy().astype(np.float64)
    ok = ~np.isnan(v)
    assert np.array_equal(of.decode(codes)[ok], v[ok]) and ok.sum() == 254
    x = np.random.default_rng(5).uniform(-1, 1, 20000) * 2.0 ** np.random.default_rng(6).uniform(-12, 8.8, 20000)
    x = np.concatenate([x.clip(-448, 448), v[ok], (v[ok][:-1] + v[ok][1:]) / 2]).astype(np.float32)
    assert np.array_equal(of.e4m3(x), torch.from_numpy(x).to(F8).float().numpy())


def test_oracle_by_hand():
    x = np.zeros((1, 144))
    x[0, :3], x[0, 130] = (448.0, -17.0, 3.0), 7.0
    t, c, s = of.quantize(x)
    assert s.tolist() == [[1.0, np.float32(7.0) / np.float32(448.0)]] and c[0, 130] == 448.0 and c[0, 1] == -16.0 and c[0, 2] == 3.0
    w, sw = np.zeros((1, 144)), np.array([[2.0, 4.0]], np.float32)
    w[0, 0], w[0, 130] = 0.5, 1.0
    u, _ = of.product(c, s, w, sw)
    assert u[0, 0] == 448.0 * 0.5 * 2.0 + 448.0 * 4.0 * float(s[0, 1])
    ids, weights = of.route(np.array([[0.0, 1.0, 1.0, -np.inf], [-np.inf] * 4], np.float32), 4)
    assert ids.tolist() == [[1, 2, 0, -1], [-1] * 4] and abs(weights[0].sum() - 1) < 1e-12 and not weights[1].any()
    ids, _ = of.route(np.array([[9.0, 0.0, 1.0, 1.5]], np.float32), 2, np.array([0, 0, 5.0, 5.0], np.float32), groups=2, top_groups=1)
    assert ids.tolist() == [[3, 2]]
