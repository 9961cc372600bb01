"""Rows of the block table and of the positions that share memory (expanded
tensors): the stride goes to the C ABI as it is, through both ways of
marshalling, and a call gives what it gives for a copy of the rows."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2607_29221_amd import _lib
from paper_2607_29221_amd import mosaic as m
from tests.cache_util import DT, TYPES, clone, make_cache, same_bits, seeded

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="CPU-only sanitizer build")
def test_strides_under_sanitizers(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    msg = tmp_path / "message.cpp"
    msg.write_text('#include "%s/paper_2607_29221_amd/csrc/abi_common.h"\n'
                   'extern "C" const char* mosaic_last_error_message(void) { return mosaic::g_last_error.c_str(); }\n'
                   % ROOT)
    objs = []
    for src in ("paper_2607_29221_amd/csrc/abi_cache.cpp", "tests/cache_stub_launchers.cpp",
                "tests/cache_sanitize_strides.cpp", str(msg)):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-g"] + SAN +
                       ["-c", os.path.join(ROOT, src), "-o", objs[-1]], check=True, capture_output=True)
    exe = str(tmp_path / "strides_san")
    subprocess.run([HIPCC] + SAN + objs + ["-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0",
                                UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"))
    assert r.returncode == 0 and "PASS" in r.stdout, r.stdout + r.stderr
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr


class _Recorder:
    """Stands in for the native marshalling (declines) and for the library
    (keeps the strides that it is handed)."""

    def __init__(self):
        self.ldt = self.ldp = None

    def cache_append(self, *args):
        return None

    def _struct(self, arg, kind):
        return ctypes.cast(arg, ctypes.POINTER(kind)).contents

    def mosaic_cache_append(self, cache, *args):
        self.ldt = self._struct(cache, _lib.MosaicKvCache).ldt
        self.ldp = self._struct(args[6], _lib.MosaicRotary).ldp
        return 0


@pytest.mark.parametrize("batch", (1, 3))
@pytest.mark.parametrize("axes", (1, 3))
def test_strides_are_passed_on(monkeypatch, batch, axes):
    """On host tensors, with the library replaced: a longer stride would read
    past the tensors' storage."""
    rec = _Recorder()
    monkeypatch.setattr(m, "_b", rec)
    monkeypatch.setattr(m._lib, "load", lambda: rec)
    monkeypatch.setattr(m, "_stream", lambda: 0)
    monkeypatch.setattr(m, "_device_tensor", lambda *args: None)
    c = m.KVCache.empty(batch, 40, 2, 64, page_size=16, device="cpu")
    table = m.Rotary.frequencies(16, 6, device="cpu")
    x, q = torch.zeros(batch, 512), torch.zeros(batch, 256)
    places = torch.zeros(batch, dtype=torch.int32)

    def call(block_table, positions):
        m.mosaic_cache_append(m.KVCache(c.k, c.v, block_table, c.state), x, 4, q,
                              rotary=m.Rotary(table, [6] if axes == 1 else [2, 2, 2], positions))
        return rec.ldt if batch > 1 else None, rec.ldp if axes > 1 else None

    wide = torch.zeros((batch, 7), dtype=torch.int32)
    assert call(wide[:, :3], torch.zeros((axes, 9), dtype=torch.int32)[:, :batch]) == \
        (7 if batch > 1 else None, 9 if axes > 1 else None)
    assert call(wide[:1, :3].expand(batch, 3), places.expand(axes, batch)) == \
        (0 if batch > 1 else None, 0 if axes > 1 else None)


def _ways(monkeypatch, native):
    """The marshalling under test: the native one, or ctypes alone."""
    if not native:
        class Declines:
            def cache_append(self, *args):
                return None
            cache_attend = cache_evict = cache_append
        monkeypatch.setattr(m, "_b", Declines())


@pytest.mark.gpu
@pytest.mark.parametrize("native", (True, False))
@pytest.mark.parametrize("act,cache", TYPES)
def test_places_shared_by_all_axes(monkeypatch, native, act, cache):
    _ways(monkeypatch, native)
    old = make_cache((3, 40, 17), 2, 64, 16, cache, 5, room=8, evicts=True)
    starts = torch.tensor([0, 2, 2, 7], dtype=torch.int32, device="cuda")
    x = torch.randn((7, 8 * 64), generator=seeded(6), device="cuda").to(DT[act])
    table = m.Rotary.frequencies(60, 32)
    # what lies behind the one row of places is another one
    rows = torch.tensor([[7, 1, 59, 30, 31, 32, 33], [40, 41, 42, 43, 44, 45, 46], [9] * 7], dtype=torch.int32,
                        device="cuda")
    got = []
    for places in (rows[:1].expand(3, 7), rows[:1].repeat(3, 1), rows[0].expand(4, 7)):
        c, q = clone(old), torch.empty((7, 256), dtype=DT[act], device="cuda")
        m.mosaic_cache_append(c, x, 4, q, starts=starts, rotary=m.Rotary(table, [8, 12, 12], places))
        got.append((q, c.k, c.v, c.state))
    for other in (got[0], got[2]):
        assert all(same_bits(a, b) for a, b in zip(other, got[1]))


@pytest.mark.gpu
@pytest.mark.parametrize("native", (True, False))
@pytest.mark.parametrize("act,cache", TYPES)
def test_pages_shared_by_all_sequences(monkeypatch, native, act, cache):
    """Several queries over one prefix; writing through the shared table is refused."""
    _ways(monkeypatch, native)
    c = make_cache((300, 280, 1), 2, 64, 16, cache, 15, evicts=True)
    q = torch.randn((3, 4 * 64), generator=seeded(16), device="cuda").to(DT[act])
    state = torch.tensor([[300, 77, 0], [300, 77, 0]], dtype=torch.int32, device="cuda")
    outs = []
    for table in (c.block_table[:1].expand(3, -1), c.block_table[:1].repeat(3, 1)):
        shared = m.KVCache(c.k, c.v, table, state, c.weights, c.order)
        out = torch.full_like(q, float("nan"))
        m.mosaic_cache_attend(shared, q, 4, out)
        outs.append(out)
    assert torch.equal(*outs) and not outs[0][2].any() and outs[0][:2].isfinite().all()
    shared = m.KVCache(c.k, c.v, c.block_table[:1].expand(3, -1), state, c.weights, c.order)
    before = clone(shared)
    for call in (lambda: m.mosaic_cache_attend(shared, q, 4, outs[0], accumulate=True),
                 lambda: m.mosaic_cache_append(shared, torch.zeros((3, 512), device="cuda"), 4, q.float()),
                 lambda: m.mosaic_cache_evict(shared, 20, 3)):
        with pytest.raises(m.MosaicError) as e:
            call()
        assert e.value.status == m.STATUS_INVALID_ARG
    assert same_bits(shared.k, before.k) and same_bits(shared.weights, before.weights)
    # one sequence shares its table with nobody
    one = m.KVCache(c.k, c.v, c.block_table[0].expand(1, -1), state[:, :1].contiguous(), c.weights, c.order)
    m.mosaic_cache_attend(one, q[:1], 4, outs[0][:1], accumulate=True)


@pytest.mark.gpu
@pytest.mark.parametrize("native", (True, False))
def test_rows_that_overlap_are_refused(monkeypatch, native):
    """A stride between 0 and the row's length."""
    _ways(monkeypatch, native)
    c = make_cache((30, 20, 10), 2, 64, 16, "bf16", 25, room=2)
    q = torch.zeros((3, 256), device="cuda")
    flat = torch.zeros(64, dtype=torch.int32, device="cuda")
    overlapping = m.KVCache(c.k, c.v, flat.as_strided((3, 2), (1, 1)), c.state)
    with pytest.raises(m.MosaicError) as e:
        m.mosaic_cache_attend(overlapping, q, 4, torch.empty_like(q))
    assert e.value.status == m.STATUS_INVALID_ARG
    rotary = m.Rotary(m.Rotary.frequencies(8, 32), [16, 16], flat.as_strided((2, 3), (1, 1)))
    with pytest.raises(m.MosaicError) as e:
        m.mosaic_cache_append(c, torch.zeros((3, 512), device="cuda"), 4, q, rotary=rotary)
    assert e.value.status == m.STATUS_INVALID_ARG


def test_places_of_one_token_have_no_stride(monkeypatch):
    """A token's places as a column: between its only entry and the next lies
    nothing that is read."""
    rec = _Recorder()
    monkeypatch.setattr(m, "_b", rec)
    monkeypatch.setattr(m._lib, "load", lambda: rec)
    monkeypatch.setattr(m, "_stream", lambda: 0)
    monkeypatch.setattr(m, "_device_tensor", lambda *args: None)
    c = m.KVCache.empty(1, 40, 2, 64, page_size=16, device="cpu")
    places = torch.zeros((1, 3), dtype=torch.int32).t()
    assert places.stride() == (1, 3)
    m.mosaic_cache_append(c, torch.zeros(1, 512), 4, torch.zeros(1, 256),
                          rotary=m.Rotary(m.Rotary.frequencies(16, 6, device="cpu"), [2, 2, 2], places))
    assert rec.ldp == 1


@pytest.mark.gpu
@pytest.mark.parametrize("native", (True, False))
def test_places_of_one_token_as_a_column(monkeypatch, native):
    _ways(monkeypatch, native)
    old = make_cache((7,), 2, 64, 16, "bf16", 35, room=2)
    x = torch.randn((1, 512), generator=seeded(36), device="cuda")
    column = torch.tensor([[3, 11, 29]], dtype=torch.int32, device="cuda").t()
    got = []
    for places in (column, column.contiguous()):
        c, q = clone(old), torch.empty((1, 256), device="cuda")
        m.mosaic_cache_append(c, x, 4, q, rotary=m.Rotary(m.Rotary.frequencies(32, 32), [8, 12, 12], places))
        got.append((q, c.k, c.v))
    assert all(same_bits(a, b) for a, b in zip(*got))


@pytest.mark.gpu
def test_native_takes_places_of_one_token_as_a_column():
    c = make_cache((7,), 2, 64, 16, "bf16", 45, room=2)
    rotary = m.Rotary(m.Rotary.frequencies(32, 32), [8, 12, 12],
                      torch.tensor([[3, 11, 29]], dtype=torch.int32, device="cuda").t())
    x, q = torch.zeros((1, 512), device="cuda"), torch.zeros((1, 256), device="cuda")
    assert m._native().cache_append(c, x, 4, q, None, rotary, None) == 0
    torch.cuda.synchronize()
