"""Where there are several devices every call refuses a tensor of another one than the current, by whichever way its arguments go: the binding's
general path, the extension module through attributes, and a cache or a packed tensor that a call is given.  Without a GPU."""
import ctypes
import importlib.machinery
import importlib.util
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from paper_2504_14152_amd import build, fgmp  # noqa: E402
from test_layer_abi import BF, I32, VP, _Tensor  # noqa: E402


class _On(_Tensor):
    """What the binding asks of a tensor of device `device`."""

    def __init__(self, device, at, *shape, **more):
        super().__init__(at, shape, **more)
        self.device, self.asked = device, 0

    def get_device(self):
        self.asked += 1
        return self.device

    def stride(self, i=None):
        return self._stride if i is None else self._stride[i]

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)


def _own_module():
    """An extension module of the test's own, that looks into no tensors."""
    fgmp.lib()
    loader = importlib.machinery.ExtensionFileLoader("_fgmp_call", build.CALL)
    module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_fgmp_call", loader))
    loader.exec_module(module)
    return module


CURRENT = 1


@pytest.fixture
def several():
    """The extension module as it is where there are several devices, the current one being CURRENT; calls are counted."""
    module = _own_module()
    module.look_into_tensors(0)
    module.current_device(lambda: CURRENT)
    called = []
    yield module, called
    module.current_device(None)
    fgmp._load_call.cache_clear()          # (what the module keeps is the process's: set up again)
    fgmp._load_call()


def _told(module, called, name, types, *given):
    f = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: called.append(name) or 0)
    return getattr(module, name)(ctypes.cast(f, VP).value, types, *given, 0x77)


def _calls(device_of):
    """Every call through the extension module; `device_of(i)`: the device of the i-th tensor, or cache, of the call."""
    number = iter(range(99))

    def t(at, *shape, **more):
        return _On(device_of(next(number)), at, *shape, **more)

    struct = fgmp._CacheStruct()

    def cache():
        return (ctypes.addressof(struct), 2, 3, 64, 40, BF, device_of(next(number)))

    yield "tree_attention", (t(16, 2, 5, 6, 64, dtype=BF), t(48, 2, 5, 3, 64, dtype=BF), t(64, 2, 5, 3, 64, dtype=BF), cache(), t(80, 2, 5, 1, dtype=torch.int64),
                             t(96, 2, dtype=I32), 0.25, 33, t(32, 2, 5, 6, 64, dtype=BF), t(112, 2, 5, 6), t(128, 999, dtype=torch.uint8))
    number = iter(range(99))
    yield "attention_weights", (t(16, 2, 5, 6, 64, dtype=BF), t(32, 2, 5, 6), cache(), t(48, 2, 3, 50), t(64, 2, 4, dtype=I32), t(80, 2, dtype=I32), 0.5, 0, t(96, 2, 3, 50))
    number = iter(range(99))
    yield "cache_append", (t(16, 2, 5, 3, 64), t(32, 2, 5, 3, 64), cache(), t(64, 2, 4, dtype=I32), t(48, 2, dtype=I32), t(64, 2, 5, dtype=I32), t(80, 2, 3, 41, dtype=I32),
                           t(96, 2, 3, 41), t(112, 2, dtype=I32))
    number = iter(range(99))
    yield "cache_evict", (cache(), t(16, 2, 3, 40), t(32, 2, 3, 40, dtype=I32), t(48, 2, dtype=I32), 30, 4, 5, t(64, 2, 3, 40), t(80, 2, 3, 40, dtype=I32), t(96, 2, dtype=I32),
                          t(112, 77, dtype=torch.uint8))
    number = iter(range(99))
    yield "block_norm", (t(16, 5, 32, dtype=BF), t(32, 5, 32), t(48, 3, 32), 2, 1, *(t(200 + 16 * i, 32) for i in range(4)), 1, 0.5, 0.25, 2, t(64, 5, 32, dtype=BF), t(80, 5, 32))
    number = iter(range(99))
    yield "quant_cache_attention", (t(16, 2, 5, 6, 64, dtype=BF), None, None, cache(), None, None, 0.25, 33, t(32, 2, 5, 6, 64, dtype=BF), t(112, 2, 5, 6), t(128, 999, dtype=torch.uint8))
    number = iter(range(99))
    yield "quant_cache_append", (t(16, 2, 5, 3, 64), t(32, 2, 5, 3, 64), cache(), t(80, 2, 4, dtype=I32), t(48, 2, dtype=I32), t(64, 2, dtype=I32))
    number = iter(range(99))
    yield "quant_cache_read", (cache(), 7, t(16, 2, 33, 3, 64), t(32, 2, 33, 3, 64))
    number = iter(range(99))
    yield "rotate_heads", (t(16, 2, 5, 6, 64), t(32, 2, 5, 3, 64), t(48, 2, 5, 3, 64), t(64, 2, 5, 3, dtype=I32), t(80, 30), t(96, 30, dtype=I32), t(112, 64), t(112, 64), 1, 0.5, True,
                           t(128, 2, 5, 6, 64, dtype=BF), t(144, 2, 5, 3, 64, dtype=BF), t(160, 2, 5, 3, 64, dtype=BF))
    number = iter(range(99))
    yield "verify_drafts", (t(16, 2, 5, 50), t(32, 2, 5, dtype=I32), t(48, 2, 5), t(64, 2, 4, 50), None, t(80, 2, dtype=I32), t(96, 2, 5, dtype=I32), t(112, 2, dtype=I32),
                            t(128, 2, dtype=I32), t(144, 77, dtype=torch.uint8))


def test_the_extension_leaves_tensors_of_another_device_to_the_general_path(several):
    module, called = several
    names = []
    for name, given in _calls(lambda i: CURRENT):
        assert _told(module, called, name, fgmp._TYPES, *given) == 0 and called == [name], name
        names.append((name, sum(isinstance(x, (_On, tuple)) for x in given)))
        called.clear()
    for name, count in names:
        for other in range(count):
            given = dict(_calls(lambda i: CURRENT if i != other else 0))[name]
            assert _told(module, called, name, fgmp._TYPES, *given) is None and called == [], (name, other)


def test_a_cache_that_does_not_say_its_device_is_left_to_the_general_path(several):
    module, called = several
    given = dict(_calls(lambda i: CURRENT))["quant_cache_read"]
    assert _told(module, called, "quant_cache_read", fgmp._TYPES, given[0][:6], *given[1:]) is None and called == []


def test_where_there_is_one_device_none_is_asked_for_it():
    fgmp.lib()
    if fgmp._several_devices():
        pytest.skip("there are several")
    for name, given in _calls(lambda i: 5):
        called = []
        assert _told(fgmp._call, called, name, fgmp._TYPES, *given) == 0 and called == [name], name
        assert not any(x.asked for x in given if isinstance(x, _On))


FUSED = ("X", "fisher", "w", "out", "workspace")


@pytest.mark.parametrize("other", [None, *FUSED])
def test_the_fused_call_does_the_same(several, other):
    module, called = several

    def t(name, at, *shape):
        return _On(0 if name == other else CURRENT, at, *shape)

    X, f, out, ws = t("X", 16, 3, 32), t("fisher", 32, 32), t("out", 48, 3, 40), t("workspace", 80, 12345)
    w = fgmp.Packed(t("w", 64, 999), 40, 32)
    e = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: called.append(1) or 0)
    rc = module.quant_gemm_fused(ctypes.cast(e, VP).value, torch.float32, BF, X, f, 0.25, 1.5, w, out, ws, 0x77)
    assert (rc, called) == ((0, [1]) if other is None else (None, []))


@pytest.mark.parametrize("host", FUSED)
def test_the_fused_call_leaves_tensors_of_the_host_to_the_general_path(host):
    fgmp.lib()

    def t(name, at, *shape):
        return _On(0, at, *shape, cuda=name != host)

    called = []
    X, f, out, ws = t("X", 16, 3, 32), t("fisher", 32, 32), t("out", 48, 3, 40), t("workspace", 80, 12345)
    w = fgmp.Packed(t("w", 64, 999), 40, 32)
    e = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: called.append(1) or 0)
    assert fgmp._call.quant_gemm_fused(ctypes.cast(e, VP).value, torch.float32, BF, X, f, 0.25, 1.5, w, out, ws, 0x77) is None and called == []


# ---- the general path ----

@pytest.fixture
def two_devices(monkeypatch):
    monkeypatch.setattr(fgmp, "_several_devices", lambda: True)
    monkeypatch.setattr(fgmp, "_current_device", lambda: CURRENT)
    monkeypatch.setattr(fgmp, "_stream", lambda: 0)
    fgmp.lib()
    monkeypatch.setattr(fgmp, "_call", None)


class _Real(torch.Tensor):
    """A CPU tensor that says it is of device `of` (-1: the host)."""
    of = CURRENT

    @property
    def is_cuda(self):
        return self.of >= 0

    def get_device(self):
        return self.of


def _real(device, t):
    t = t.as_subclass(_Real)
    t.of = device
    return t


PRODUCTS = ["quantize_weights", "quantize_weights_clip", "quantize_activations", "gemm", "quant_gemm_fused", "quant_gemm_fused_static_scratch", "quant_gemm_fused_packed_out",
            "unpack_canonical", "dequantize_f16", "quantize_dequantize_f16", "packed_info", "threshold_for_fraction", "threshold_for_fraction_multi"]
GIVEN = {"quantize_weights": "X f packed", "quantize_weights_clip": "X f packed", "quantize_activations": "X f packed", "gemm": "packed weights out workspace",
         "quant_gemm_fused": "X f weights out workspace", "quant_gemm_fused_static_scratch": "X f weights out", "quant_gemm_fused_packed_out": "X f weights fn packed workspace",
         "unpack_canonical": "packed", "dequantize_f16": "packed out", "quantize_dequantize_f16": "X f out", "packed_info": "packed", "threshold_for_fraction": "X",
         "threshold_for_fraction_multi": "X f"}


def _product(name, where):
    """A call whose tensor `where` is of another device than all others."""
    class Refused(Exception):
        pass

    def t(what, *shape, dtype=torch.float32):
        return _real(where[1] if what == where[0] else CURRENT, torch.zeros(*shape, dtype=dtype))

    X, f, fn, out, ws = t("X", 3, 32), t("f", 32), t("fn", 32), t("out", 3, 32), t("workspace", 64, dtype=torch.uint8)
    packed, weights = fgmp.Packed(t("packed", 99, dtype=torch.uint8), 3, 32), fgmp.Packed(t("weights", 99, dtype=torch.uint8), 32, 32)
    return {"quantize_weights": lambda: fgmp.quantize_weights(X, f, 0.5, 1.0, out=packed), "quantize_weights_clip": lambda: fgmp.quantize_weights_clip(X, f, 0.5, 1.0, out=packed),
            "quantize_activations": lambda: fgmp.quantize_activations(X, f, 0.5, 1.0, out=packed), "gemm": lambda: fgmp.gemm(packed, weights, out, ws),
            "quant_gemm_fused": lambda: fgmp.quant_gemm_fused(X, f, 0.5, 1.0, weights, out, ws),
            "quant_gemm_fused_static_scratch": lambda: fgmp.quant_gemm_fused_static_scratch(X, f, 0.5, 1.0, weights, out),
            "quant_gemm_fused_packed_out": lambda: fgmp.quant_gemm_fused_packed_out(X, f, 0.5, 1.0, weights, fn, 0.5, 1.0, out=packed, workspace=ws),
            "unpack_canonical": lambda: fgmp.unpack_canonical(packed), "dequantize_f16": lambda: fgmp.dequantize_f16(packed, out),
            "quantize_dequantize_f16": lambda: fgmp.quantize_dequantize_f16(X, f, 0.5, 1.0, out), "packed_info": lambda: fgmp.packed_info(packed),
            "threshold_for_fraction": lambda: fgmp.threshold_for_fraction(X, 0.5), "threshold_for_fraction_multi": lambda: fgmp.threshold_for_fraction_multi([X, f], 0.5)}[name]


@pytest.mark.parametrize("name", PRODUCTS)
def test_products_and_quantizers_refuse(two_devices, monkeypatch, name):
    class Library:
        def __getattr__(self, entry):
            raise AssertionError(f"{entry} called")

    monkeypatch.setattr(fgmp, "lib", Library)
    for what in GIVEN[name].split():
        with pytest.raises(fgmp.FgmpError, match="current device, 1"):
            _product(name, (what, 0))()
        with pytest.raises(fgmp.FgmpError, match="on the GPU"):
            _product(name, (what, -1))()
    with pytest.raises(AssertionError, match="called"):        # (all on the current device: handed on)
        _product(name, (None, 0))()


def _quant_cache(device):
    def t(*shape, dtype):
        return _real(device, torch.zeros(*shape).to(dtype))

    return fgmp.QuantCache(t(4, 32, 2, 64, dtype=torch.float8_e4m3fn), t(4, 32, 2, 64, dtype=torch.float8_e4m3fn), t(4, 2, 32, dtype=torch.uint8), t(4, 2, 32, dtype=torch.uint8),
                           t(2, dtype=torch.int32), t(2, 2, dtype=torch.int32))


def _cache(device):
    def t(*shape, dtype=BF):
        return _real(device, torch.zeros(*shape).to(dtype))

    return fgmp.Cache(t(4, 32, 2, 64), t(4, 32, 2, 64), t(2, dtype=torch.int32), t(2, 2, dtype=torch.int32))


@pytest.mark.parametrize("make", [_cache, _quant_cache])
def test_a_cache_of_another_device_is_refused_by_the_calls(two_devices, monkeypatch, make):
    """The cache was made while its device was the current one; now another is."""
    monkeypatch.setattr(fgmp, "_current_device", lambda: 0)
    c = make(0)
    assert c._handle[6] == 0
    monkeypatch.setattr(fgmp, "_current_device", lambda: CURRENT)
    q = _real(CURRENT, torch.zeros(2, 1, 2, 64, dtype=BF))
    lse, weights, n = (_real(CURRENT, torch.zeros(*s, dtype=d)) for s, d in (((2, 1, 2), torch.float32), ((2, 2, 64), torch.float32), ((2,), torch.int32)))
    slots = _real(CURRENT, torch.zeros(2, 2, 64, dtype=torch.int32))
    calls = [lambda: fgmp.tree_attention(q, q, q, c), lambda: fgmp.cache_append(q, q, c)]
    if make is _cache:
        calls += [lambda: fgmp.attention_weights(q, lse, c, weights), lambda: fgmp.cache_evict(c, weights, slots, n, 10)]
    else:
        calls += [lambda: fgmp.cache_read(c)]
    for call in calls:
        with pytest.raises(fgmp.FgmpError, match="current device, 1"):
            call()
    with pytest.raises(fgmp.FgmpError, match="current device, 1"):
        c.lengths = n                            # (on the current device, the cache is not)
