"""Host side of the cached decoding (no GPU needed): the C ABI's validation
under AddressSanitizer and UndefinedBehaviorSanitizer with the launchers
replaced, the Python layer's refusals, and the oracle's own checks."""
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import _lib
from paper_2607_29221_amd import mosaic as m

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"
SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="CPU-only sanitizer build")
def test_validation_under_sanitizers(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    objs = []
    for src in ("paper_2607_29221_amd/csrc/abi_cache.cpp", "tests/cache_stub_launchers.cpp",
                "tests/cache_sanitize_driver.cpp"):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-g"] + SAN +
                       ["-c", os.path.join(ROOT, src), "-o", obj], check=True, capture_output=True)
        objs.append(obj)
    # mosaic_last_error_message lives in the other part of the ABI layer
    msg = tmp_path / "message.cpp"
    msg.write_text('#include "%s/paper_2607_29221_amd/csrc/abi_common.h"\n'
                   'extern "C" const char* mosaic_last_error_message(void) { return mosaic::g_last_error.c_str(); }\n'
                   % ROOT)
    obj = str(tmp_path / "message.o")
    subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-g"] + SAN +
                   ["-c", str(msg), "-o", obj], check=True, capture_output=True)
    exe = str(tmp_path / "cache_san")
    subprocess.run([HIPCC] + SAN + objs + [obj, "-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0",
                                UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"))
    assert r.returncode == 0 and "PASS" in r.stdout, r.stdout + r.stderr
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr


def test_structs_match_the_header():
    """Sizes of the structs as a C compiler lays them out."""
    import ctypes
    assert ctypes.sizeof(_lib.MosaicKvCache) == 10 * 8 + 6 * 4
    assert ctypes.sizeof(_lib.MosaicRotary) == 4 * 8 + 6 * 4
    assert _lib.MosaicKvCache.dtype.offset == 80 and _lib.MosaicRotary.naxes.offset == 32


def test_host_tensors_are_refused():
    c = m.KVCache.empty(2, 40, 2, 64, page_size=16, evicts=True, device="cpu")
    q = torch.zeros(2, 256)
    with pytest.raises(ValueError):
        m.mosaic_cache_append(c, torch.zeros(2, 512), 4, q)
    with pytest.raises(ValueError):
        m.mosaic_cache_attend(c, q, 4, torch.zeros(2, 256))
    with pytest.raises(ValueError):
        m.mosaic_cache_evict(c, 10, 2)


def test_empty_cache():
    c = m.KVCache.empty(3, 100, 2, 64, page_size=32, evicts=True, device="cpu")
    assert c.batch == 3 and c.slots == 128 and c.k.shape == (12, 2, 32, 64)
    assert sorted(c.block_table.flatten().tolist()) == list(range(12)) and not c.state.any()


def test_table_of_angles():
    t = m.Rotary.frequencies(50, 3, base=100.0, device="cpu")
    assert t.shape == (50, 6) and t.dtype == torch.float32
    a = 49 * 100.0 ** (-2 / 3)
    assert abs(float(t[49, 2]) - np.cos(a)) < 1e-7 and abs(float(t[49, 5]) - np.sin(a)) < 1e-7


def test_oracle_attention_of_one_and_none():
    v = np.array([[1.0, 2.0]])
    out, p = oc.attend([[3.0, 4.0]], [[5.0, 6.0]], v, 0.1)
    assert np.array_equal(out, v) and p.tolist() == [[1.0]]
    out, p = oc.attend([[3.0, 4.0]], np.zeros((0, 2)), np.zeros((0, 2)), 0.1)
    assert not out.any() and p.shape == (1, 0)


def test_oracle_rotation_keeps_products():
    """Turning query and key by the same number of further places leaves their
    product alone, and a pair keeps its length."""
    r = np.random.default_rng(1)
    table = m.Rotary.frequencies(64, 4, device="cpu").numpy()
    x = r.standard_normal((2, 1, 10))
    for interleaved in (False, True):
        dots = []
        for shift in (0, 13):
            y = oc.rotate(x, table, np.array([[5 + shift, 20 + shift]] * 2), [1, 3], interleaved)
            dots.append(float(y[0, 0] @ y[1, 0]))
            assert np.allclose((y ** 2).sum(), (x ** 2).sum(), rtol=1e-6)
        assert abs(dots[0] - dots[1]) < 1e-5
        assert np.array_equal(y[..., 8:], x[..., 8:])


def test_oracle_eviction_by_hand():
    w = [5.0, 0.0, 3.0, 3.0, 1.0, 0.0]
    assert oc.evict(w, [0, 1, 2, 3, 4, 5], 6, 6, 0) == [0, 1, 2, 3, 4, 5]
    assert oc.evict(w, [0, 1, 2, 3, 4, 5], 6, 3, 0) == [0, 3, 2]        # 3 comes to the free slot 1
    assert oc.evict(w, [0, 1, 2, 3, 4, 5], 6, 3, 1) == [0, 5, 2]        # the latest stays; the tie goes to slot 2
    assert oc.evict(w, [0, 5, 2, 3, 4, 1], 6, 2, 1) == [0, 1]           # the latest is in slot 1
    assert oc.evict([float("nan"), 1.0, -1.0], [0, 1, 2], 9, 2, 0) == [2, 1]
