"""Where the binding's calls take the memory of the tensors that they make for themselves: from the stream that they run on.  Without a GPU: the library
is a stub, and streams are names.  And that what they are given is on the current device."""
import contextlib

import pytest
import torch

import paper_2511_11446_amd as ql


class _OnGpu(torch.Tensor):
    """A CPU tensor that says it is on the GPU, and which streams use it."""

    is_cuda = True

    def get_device(self):
        return 0

    def record_stream(self, stream):
        self.__dict__.setdefault("used_on", []).append(stream)


class _Stream:
    def __init__(self, handle):
        self.cuda_stream = handle

    def __eq__(self, other):
        return self.cuda_stream == other.cuda_stream

    def __hash__(self):
        return self.cuda_stream


CURRENT = _Stream(0)


class _Library:
    """Every call of the library: remembered, and well; sizes in bytes are 1000."""

    def __getattr__(self, name):
        class Call:
            def __call__(self, *args):
                return 1000 if name.endswith("_bytes") else 0

        call = Call()
        setattr(self, name, call)
        return call


@pytest.fixture
def made(monkeypatch):
    """The tensors that calls make, each with the stream whose memory it has."""
    tensors, active, empty = [], [CURRENT], torch.empty

    @contextlib.contextmanager
    def stream(s):
        active.append(s)
        yield
        active.pop()

    def on(*shape, dtype=None, device=None):
        t = empty(*shape, dtype=dtype).as_subclass(_OnGpu)
        t.memory_of = active[-1]
        tensors.append(t)
        return t

    library = _Library()
    monkeypatch.setattr(ql, "lib", lambda: library)
    monkeypatch.setattr(ql, "_current", lambda: 0)
    monkeypatch.setattr(ql, "_raw_stream", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch, "empty", on)
    for name, value in (("stream", stream), ("Stream", _Stream), ("ExternalStream", _Stream), ("current_stream", lambda *a: active[-1]), ("default_stream", lambda *a: CURRENT)):
        monkeypatch.setattr(torch.cuda, name, value)
    return tensors


def _t(*shape, dtype=torch.float16):
    return torch.zeros(shape, dtype=dtype).as_subclass(_OnGpu)


def _cache():
    return ql.KvCache8(_t(2, 2, 64, 64, dtype=torch.int8), _t(2, 2, 1, 64, 64, dtype=torch.int8), _t(2, 2, 1, dtype=torch.float32), _t(2, 2, 1, dtype=torch.float32))


def _ints(*shape):
    return _t(*shape, dtype=torch.int32)


W8, S8, W4 = _t(32, 256, dtype=torch.int8), _t(32, dtype=torch.float32), _t(32, 128, dtype=torch.uint8)
CALLS = {
    "attention_f16": lambda **kw: ql.attention_f16(_t(8, 2, 64), _t(8, 2, 64), _t(8, 2, 64), **kw),
    "attention_kv8": lambda **kw: ql.attention_kv8(_t(8, 2, 64), _cache(), _ints(1, 2), _ints(1), **kw),
    "daq_kv_append": lambda **kw: ql.daq_kv_append(_cache(), _t(8, 2, 64), _t(8, 2, 64), _ints(1, 2), _ints(1), q=_t(8, 2, 64), **kw),
    "daq_quantize": lambda **kw: ql.daq_quantize(_t(8, 256), 4, **kw),
    "daq_quantize_rowmax": lambda **kw: ql.daq_quantize_rowmax(_t(8, 256), 4, _ints(8), **kw),
    "daq_quantize_ln": lambda **kw: ql.daq_quantize_ln(_t(8, 256), 4, want_h=True, **kw),
    "daq_quantize_cg": lambda **kw: ql.daq_quantize_cg(_t(8, 256), 4, 64, **kw),
    "daq_quantize_robust": lambda **kw: ql.daq_quantize_robust(_t(8, 256), 4, **kw),
    "qlinear_grouped": lambda **kw: ql.qlinear_grouped(_t(8, 256), 4, W8, _t(32, 4), 64, act_group=64, debug=True, **kw),
    "qlinear_fused": lambda **kw: ql.qlinear_fused(_t(8, 256), 4, W8, S8, **kw),
    "qlinear_f16": lambda **kw: ql.qlinear_f16(_t(8, 256), _t(32, 256), **kw),
    "qlinear_w8a8": lambda **kw: ql.qlinear_w8a8(_t(8, 256), 4, W8, S8, debug=True, **kw),
    "qlinear_w4a8": lambda **kw: ql.qlinear_w4a8(_t(8, 256), 4, W4, _t(32, 4), group=64, debug=True, **kw),
    "qgemm_w8a8": lambda **kw: ql.qgemm_w8a8(_t(8, 256, dtype=torch.int8), S8, 4, W8, S8, **kw),
    "qgemm_w4a8": lambda **kw: ql.qgemm_w4a8(_t(8, 256, dtype=torch.int8), S8, 4, W4, _t(32, 4), group=64, **kw),
    "prepack_w4": lambda **kw: ql.prepack_w4(W4, **kw),
}


def _tensors(out):
    return [t for x in (out.values() if isinstance(out, dict) else out if isinstance(out, tuple) else [out]) for t in [x] if isinstance(t, torch.Tensor)]


@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("stream, handle", [(_Stream(0x50), 0x50), (0x50, 0x50), (0, 0)])
def test_memory_is_of_the_stream_that_the_call_runs_on(name, stream, handle, made):
    returned = _tensors(CALLS[name](stream=stream))
    assert made and all(t.memory_of.cuda_stream == handle for t in made), [t.memory_of.cuda_stream for t in made]
    # what the caller gets is used on the current stream as a rule: freed, it has to wait for that one
    for t in returned:
        assert CURRENT in t.__dict__.get("used_on", []) or t.memory_of == CURRENT


@pytest.mark.parametrize("name", sorted(CALLS))
def test_without_a_stream_nothing_is_recorded(name, made):
    CALLS[name]()
    assert made and all(t.memory_of == CURRENT and "used_on" not in t.__dict__ for t in made)


class _OnTheOther(_OnGpu):
    def get_device(self):
        return 1


CACHED = {
    "attention_kv8": lambda cache, **kw: ql.attention_kv8(_t(8, 2, 64), cache, _ints(1, 2), _ints(1), **kw),
    "daq_kv_append": lambda cache, **kw: ql.daq_kv_append(cache, _t(8, 2, 64), _t(8, 2, 64), _ints(1, 2), _ints(1), **kw),
}


@pytest.mark.parametrize("name", sorted(CACHED))
@pytest.mark.parametrize("part", ["k", "v", "k_scale", "v_scale"])
def test_every_part_of_the_cache_is_on_the_current_device(name, part, made):
    here = _cache()
    parts = {p: getattr(here, p) for p in ("k", "v", "k_scale", "v_scale")}
    parts[part] = parts[part].as_subclass(_OnTheOther)
    with pytest.raises(ValueError, match="is on .* current device"):
        CACHED[name](ql.KvCache8(*parts.values()))
    CACHED[name](here)


@pytest.mark.parametrize("name", ["attention_f16", "attention_kv8", "daq_kv_append"])
def test_the_stream_is_on_the_current_device(name, made):
    s = _Stream(0x50)
    s.device_index = 1
    with pytest.raises(ValueError, match="stream is on cuda:1"):
        CALLS[name](stream=s)
    s.device_index = 0
    CALLS[name](stream=s)


@pytest.mark.parametrize("rot", [_t(0, 32, 2, dtype=torch.float32), _t(4, 0, 2, dtype=torch.float32), _t(4, 32, 3, dtype=torch.float32)])
def test_an_empty_rotation_table_is_refused(rot, made):
    """Its address is none, which would mean no rotation at all."""
    with pytest.raises(ValueError, match="rot must be"):
        ql.daq_kv_append(_cache(), _t(8, 2, 64), _t(8, 2, 64), _ints(1, 2), _ints(1), rot=rot)


@pytest.mark.parametrize("page, scale_tokens", [(64, 48), (64, 33), (128, 8), (64, 0), (96, 32), (32, 32), (64, 128), (64, -1)])
def test_an_empty_cache_has_the_scales_that_were_asked_for(page, scale_tokens, made):
    with pytest.raises(ValueError, match="page|scale_tokens"):
        ql.KvCache8.empty(4, 2, 64, page=page, scale_tokens=scale_tokens)
