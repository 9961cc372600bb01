"""k_out and v_out of mosaic_cache_read as columns of one matrix: taken where they
lie side by side, refused where they overlap."""
import os
import subprocess

import pytest
import torch

from paper_2607_29221_amd import mosaic as m
from tests import cache_util as cu
from tests import e2m1_util as eu
from tests.cache_util import DT, TYPES
from tests.test_cache_host import HIPCC, ROOT, SAN


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="CPU-only sanitizer build")
def test_side_by_side_under_sanitizers(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    msg = tmp_path / "message.cpp"
    msg.write_text('#include "%s/paper_2607_29221_amd/csrc/abi_common.h"\n'
                   'extern "C" const char* mosaic_last_error_message(void) { return mosaic::g_last_error.c_str(); }\n' % ROOT)
    objs = []
    for src in ("paper_2607_29221_amd/csrc/abi_cache.cpp", "paper_2607_29221_amd/csrc/abi_cache_norm.cpp",
                "tests/cache_stub_launchers.cpp", "tests/cache_norm_stub_launchers.cpp",
                "tests/cache_read_sanitize_driver.cpp", str(msg)):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-g"] + SAN +
                       ["-c", os.path.join(ROOT, src), "-o", objs[-1]], check=True, capture_output=True)
    exe = str(tmp_path / "read_san")
    subprocess.run([HIPCC] + SAN + objs + ["-o", exe], check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0",
                                UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1"))
    assert r.returncode == 0 and "PASS" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr


def both(c, act, gap):
    """Columns k | gap | v of one matrix, and what separate outputs get."""
    rows, width = sum(c.state[0].tolist()), c.k.shape[1] * (c.k.shape[3] if c.head_dim is None else c.head_dim)
    starts = torch.tensor([0, 40, rows], dtype=torch.int32, device="cuda")
    kv = torch.full((rows, 2 * width + gap), 7.0, dtype=DT[act], device="cuda")
    m.mosaic_cache_read(c, kv[:, :width], kv[:, width + gap:], starts=starts)
    k, v = (torch.empty((rows, width), dtype=DT[act], device="cuda") for _ in range(2))
    m.mosaic_cache_read(c, k, v, starts=starts)
    assert torch.equal(kv[:, :width], k) and torch.equal(kv[:, width + gap:], v) and (kv[:, width: width + gap] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("act", eu.ACTS)
@pytest.mark.parametrize("gap", (0, 16))
def test_rows_of_4_bits_side_by_side(act, gap):
    both(eu.make_cache((40, 33), 2, 80, 16, 5), act, gap)


@pytest.mark.gpu
@pytest.mark.parametrize("out,cache", TYPES)
def test_rows_of_16_and_32_bits_side_by_side(out, cache):
    both(cu.make_cache((40, 33), 2, 64, 16, cache, 6), out, 8)


@pytest.mark.gpu
def test_overlapping_columns_are_refused():
    c = eu.make_cache((5, 3), 2, 64, 16, 7)
    kv = torch.zeros((2, 400), device="cuda")
    for first, second in ((0, 0), (0, 124), (124, 0), (0, 300), (16, 140)):
        with pytest.raises((m.MosaicError, ValueError)):
            m.mosaic_cache_read(c, kv[:, first: first + 128], kv[:, second: second + 128])
