"""Host side of norms and of caches in 4 bits (no GPU needed): the C ABI's
validation under AddressSanitizer and UndefinedBehaviorSanitizer with the
launchers replaced, the Python layer's refusals, and the oracle's own checks."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_29221_amd import _lib
from paper_2607_29221_amd import mosaic as m
from tests.test_cache_host import HIPCC, ROOT, SAN


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="CPU-only sanitizer build")
def test_validation_under_sanitizers(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    msg = tmp_path / "message.cpp"
    msg.write_text('#include "%s/paper_2607_29221_amd/csrc/abi_common.h"\n'
                   'extern "C" const char* mosaic_last_error_message(void) { return mosaic::g_last_error.c_str(); }\n' % ROOT)
    objs = []
    for src in ("paper_2607_29221_amd/csrc/abi_cache.cpp", "paper_2607_29221_amd/csrc/abi_cache_norm.cpp",
                "tests/cache_stub_launchers.cpp", "tests/cache_norm_stub_launchers.cpp",
                "tests/cache_norm_sanitize_driver.cpp", str(msg)):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-g"] + SAN +
                       ["-c", os.path.join(ROOT, src), "-o", obj], check=True, capture_output=True)
        objs.append(obj)
    exe = str(tmp_path / "cache_norm_san")
    subprocess.run([HIPCC] + SAN + objs + ["-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0",
                                UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"))
    assert r.returncode == 0 and "PASS" in r.stdout, r.stdout + r.stderr
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr


def test_structs_match_the_header():
    assert ctypes.sizeof(_lib.MosaicQkNorm) == 2 * 8 + 8 and _lib.MosaicQkNorm.eps.offset == 16


def test_host_tensors_are_refused():
    c = m.KVCache.empty(2, 40, 2, 64, torch.uint8, page_size=16, evicts=True, device="cpu")
    q, w = torch.zeros(2, 256), torch.ones(64)
    for call in (lambda: m.mosaic_cache_append_norm(c, torch.zeros(2, 512), 4, q, m.QKNorm(w, w)),
                 lambda: m.mosaic_cache_append(c, torch.zeros(2, 512), 4, q),
                 lambda: m.mosaic_cache_read(c, torch.zeros(2, 128), torch.zeros(2, 128)),
                 lambda: m.mosaic_cache_attend(c, q, 4, torch.zeros(2, 256)), lambda: m.mosaic_cache_evict(c, 10, 2)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dim,width", ((8, 16), (16, 16), (24, 16), (32, 32), (64, 48), (72, 48), (80, 64), (128, 80), (256, 160)))
def test_empty_cache(dim, width):
    c = m.KVCache.empty(3, 100, 2, dim, torch.uint8, page_size=32, evicts=True, device="cpu")
    assert c.k.shape == (12, 2, 32, width) and c.k.dtype == torch.uint8 and c.head_dim == dim
    assert m.KVCache.row_bytes(dim) == width == oc.row_bytes(dim)


def test_oracle_codes_by_hand():
    x = np.array([[0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], [-7.0, 0.26, 0.74, 1.26, 1.74, 2.51, 3.49, 5.01],
                  [7.5, 0.5, 1.0, 1.5, 2.5, 3.5, 5.0, 7.0], [2.0 ** -130] * 8, [2.0 ** 127 * 1.9] + [2.0 ** 125] * 7,
                  [np.inf] + [1.0] * 7])
    codes, scales = oc.to_e2m1(x)
    assert scales[:, 0].tolist() == [127, 127, 128, 1, 252, 255]
    assert codes[0].tolist() == [0, 0, 2, 2, 4, 4, 6, 6]            # to even codes between two
    assert codes[1].tolist() == [15, 1, 1, 3, 3, 5, 5, 7]           # 7 is as near as it gets
    assert codes[2].tolist() == [6, 0, 1, 2, 2, 4, 4, 6]            # twice the scale: .25, .5, .75, 1.25, 1.75, 2.5, 3.5
    assert codes[4].tolist() == [7] + [2] * 7
    back = oc.unpack_e2m1(oc.pack_e2m1(codes, scales), 8)
    assert back[2].tolist() == [8.0, 0.0, 1.0, 2.0, 2.0, 4.0, 4.0, 8.0] and not back[3].any() and np.isnan(back[5]).all()


@pytest.mark.parametrize("dim", (8, 80, 128))
def test_oracle_round_trip(dim):
    """An element is off by half the distance of its codes at most, a fifth of the
    largest of its 8; what a row holds is held again the same."""
    x = np.random.default_rng(dim).standard_normal((200, dim)) * np.exp(np.random.default_rng(1).standard_normal((200, 1)) * 9)
    rows = oc.pack_e2m1(*oc.to_e2m1(x))
    y = oc.unpack_e2m1(rows, dim)
    top = np.abs(x).reshape(200, -1, 8).max(axis=-1).repeat(8, axis=-1)
    assert (np.abs(x - y) <= 0.2 * top).all() and (np.abs(x - y) <= np.maximum(np.abs(x) / 3, top / 3.5 / 4)).all()
    assert np.array_equal(oc.unpack_e2m1(oc.pack_e2m1(*oc.to_e2m1(y)), dim), y)


def test_oracle_norm():
    x = np.array([[3.0, 4.0, 0.0, 0.0]])
    assert np.allclose(oc.normalise(x, [1.0, 2.0, 1.0, 1.0], 0.0), [[1.2, 3.2, 0.0, 0.0]], rtol=1e-15)
    assert np.allclose(oc.normalise(x, [1.0] * 4, 18.75), [[0.6, 0.8, 0.0, 0.0]], rtol=1e-15)
