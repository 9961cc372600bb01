"""Every tensor of a call of the cached decoding lies on the cache's device, and
that is the current one: both ways into the C ABI, native marshalling and ctypes,
refuse a call with a single one elsewhere. No GPU needed: the tensors are host
memory that says it is device memory, and the library is replaced by functions
that do nothing."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2607_29221_amd import mosaic as m

SIZE = {torch.float32: 4, torch.int32: 4, torch.uint8: 1, torch.bfloat16: 2}


def fake(device, shape, dtype):
    """A contiguous tensor that says it lies on cuda:<device>."""
    strides = [int(np.prod(shape[i + 1:])) for i in range(len(shape))]
    memory = np.zeros(int(np.prod(shape)) * SIZE[dtype] + 64, np.uint8)
    start = (memory.ctypes.data + 63) // 64 * 64
    storage = torch._C._construct_storage_from_data_pointer(start, torch.device("cuda", device), len(memory) - 64)
    t = torch._C._construct_CUDA_Tensor_From_Storage_And_Metadata(
        {"dtype": dtype, "size": tuple(shape), "stride": tuple(strides), "storage_offset": 0}, storage)
    t.memory = memory
    assert t.device == torch.device("cuda", device) and t.data_ptr() == start
    return t


F, I = torch.float32, torch.int32
# name -> (shape, type): 3 sequences, 4 query heads on 2 of 64 elements, 5 new tokens, pages of 16
TENSORS = {"v": ((9, 2, 16, 48), torch.uint8), "block_table": ((3, 3), I), "state": ((2, 3), I), "weights": ((9, 2, 16), F),
           "order": ((9, 2, 16), I), "qkv": ((5, 512), F), "q_out": ((5, 256), F), "starts": ((4,), I), "first": ((3,), I),
           "table": ((100, 64), F), "positions": ((2, 5), I), "q_weight": ((64,), F), "k_weight": ((64,), F),
           "new_state": ((2, 3), I), "k_out": ((5, 128), F), "v_out": ((5, 128), F), "q": ((3, 256), F), "out": ((3, 256), F),
           "new_weights": ((9, 2, 16), F), "new_order": ((9, 2, 16), I), "kept": ((3, 2, 20), I)}
CACHE = ("v", "block_table", "state", "weights", "order")
CALLS = {
    "cache_append": (("qkv", "q_out", "starts", "table", "positions", "new_state"),
                     lambda c, t: (c, t["qkv"], 4, t["q_out"], t["starts"], rotary(t), t["new_state"])),
    "cache_append_norm": (("qkv", "q_out", "q_weight", "k_weight", "starts", "table", "positions", "new_state"),
                          lambda c, t: (c, t["qkv"], 4, t["q_out"], m.QKNorm(t["q_weight"], t["k_weight"]), t["starts"],
                                        rotary(t), t["new_state"])),
    "cache_read": (("k_out", "v_out", "starts", "first"), lambda c, t: (c, t["k_out"], t["v_out"], t["starts"], t["first"])),
    "cache_attend": (("q", "out"), lambda c, t: (c, t["q"], 4, t["out"], 40, 0.125, True)),
    "cache_evict": (("new_state", "new_weights", "new_order", "kept"),
                    lambda c, t: (c, 20, 2, 40, t["new_state"], t["new_weights"], t["new_order"], t["kept"])),
}


def rotary(t):
    return m.Rotary(t["table"], (20, 12), t["positions"])


def args(name, four, elsewhere=None, device=0):
    """Arguments of a call over 4 or 16 bits; the tensor ``elsewhere`` on the other device."""
    dtype = torch.uint8 if four else torch.bfloat16
    spec = dict(TENSORS, k=((9, 2, 16, 48 if four else 64), dtype), v=((9, 2, 16, 48 if four else 64), dtype))
    t = {n: fake(1 - device if n == elsewhere else device, *spec[n]) for n in ("k",) + CACHE + CALLS[name][0]}
    cache = m.KVCache(*(t[n] for n in ("k",) + CACHE), head_dim=64 if four else None)
    return CALLS[name][1](cache, t)


@pytest.fixture
def library(monkeypatch):
    """The native marshalling bound to functions that count their calls; the
    current device is number 0."""
    called, kept = [], []

    def entry(name):
        if name.endswith("_workspace"):               # *bytes = 0
            proto = ctypes.CFUNCTYPE(ctypes.c_int32, *([ctypes.c_int64] * (4 if "attend" in name else 3)),
                                     ctypes.POINTER(ctypes.c_int64))

            def call(*a):
                a[-1][0] = 0
                return 0
        else:
            proto = ctypes.CFUNCTYPE(ctypes.c_int32)

            def call():
                called.append(name)
                return 0
        kept.append(proto(call))
        return ctypes.cast(kept[-1], ctypes.c_void_p).value
    native, lib = m._native(), m._lib.load()
    native.bind(tuple(entry(n) for n in m._BOUND), lambda: 0, lambda device: 0, m._lib.MosaicRng)
    native.called = called
    yield native
    native.bind(tuple(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in m._BOUND), torch._C._cuda_getDevice,
                torch._C._cuda_getCurrentRawStream, m._lib.MosaicRng)


class _Library:
    """Stands in for the library behind the ctypes calls, and for native marshalling that declines."""

    def __init__(self):
        self.called = []

    def __getattr__(self, name):
        if name in CALLS:
            return lambda *a: None
        return lambda *a: self.called.append(name) or 0


def by_ctypes(monkeypatch, current=0):
    lib = _Library()
    monkeypatch.setattr(m, "_b", lib)
    monkeypatch.setattr(m._lib, "load", lambda: lib)
    monkeypatch.setattr(m, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: empty(*a, dtype=kw["dtype"]))
    return lib


EACH = [(name, t) for name in CALLS for t in CACHE + CALLS[name][0]]


@pytest.mark.parametrize("four", (False, True))
@pytest.mark.parametrize("name", list(CALLS))
def test_calls_on_one_device_are_made(library, monkeypatch, name, four):
    assert getattr(library, name)(*args(name, four)) == 0 and library.called == ["mosaic_" + name]
    lib = by_ctypes(monkeypatch)
    getattr(m, "mosaic_" + name)(*args(name, four))
    assert lib.called[-1] == "mosaic_" + name




@pytest.mark.parametrize("name,elsewhere", EACH)
def test_native_marshalling_declines(library, name, elsewhere):
    for four in (False, True):
        assert getattr(library, name)(*args(name, four, elsewhere=elsewhere)) is None
    assert library.called == []


@pytest.mark.parametrize("name,elsewhere", EACH)
def test_python_refuses(monkeypatch, name, elsewhere):
    lib = by_ctypes(monkeypatch)
    for four in (False, True):
        with pytest.raises(ValueError, match="another device"):
            getattr(m, "mosaic_" + name)(*args(name, four, elsewhere=elsewhere))
    assert lib.called == []


@pytest.mark.parametrize("name", list(CALLS))
def test_all_on_another_device_than_the_current_one(library, monkeypatch, name):
    for four in (False, True):
        assert getattr(library, name)(*args(name, four, device=1)) is None
    assert library.called == []
    lib = by_ctypes(monkeypatch)
    for four in (False, True):
        with pytest.raises(ValueError, match="another device"):
            getattr(m, "mosaic_" + name)(*args(name, four, device=1))
    assert lib.called == []
