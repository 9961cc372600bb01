"""How the attention over 4 bits is dealt out, by the host code of its kernel (no
GPU needed): no more workgroups than the units hold at once unless more than one
unit in 16 would idle, and no more than the workspace has room for."""
import ctypes
import os
import subprocess

import pytest

from tests.test_cache_host import HIPCC, ROOT

UNITS, LDS = 256, 160 * 1024
TYPES = ("f32", "bf16", "f16")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if os.path.exists("/dev/kfd") or not os.path.exists(HIPCC):
        pytest.skip("host-only build")
    tmp = str(tmp_path_factory.mktemp("plan"))
    obj, so = os.path.join(tmp, "probe.o"), os.path.join(tmp, "plan.so")
    subprocess.run([HIPCC, "-x", "hip", "--cuda-host-only", "-std=c++17", "-O1", "-fPIC", "-c",
                    os.path.join(ROOT, "tests", "attend_plan_probe.cpp"), "-o", obj], check=True, capture_output=True)
    subprocess.run(["objcopy", "-w", "--weaken-symbol=__hip_fatbin*", obj], check=True)      # there is no code for a device
    subprocess.run([os.environ.get("CXX", "g++"), "-shared", "-fPIC", obj,
                    os.path.join(ROOT, "tests", "hip_runtime_stubs.cpp"), "-o", so], check=True)
    lib = ctypes.CDLL(so)
    lib.attend_plan.argtypes = [ctypes.c_int] * 5 + [ctypes.c_int64, ctypes.c_int, ctypes.c_void_p]

    def call(act, batch, heads, kv, dim, max_len, accumulate):
        out = (ctypes.c_int32 * 4)()
        lib.attend_plan(TYPES.index(act), batch, heads, kv, dim, max_len, accumulate, out)
        return list(out)
    return call


@pytest.mark.parametrize("act", TYPES)
@pytest.mark.parametrize("accumulate", (False, True))
@pytest.mark.parametrize("dim", (8, 64, 72, 96, 128, 136, 256))
def test_workgroups_fit(plan, act, accumulate, dim):
    for kv in (1, 2, 4, 8):
        for group in (1, 4, 5, 8, 9, 16, 17, 32, 33, 64, 100):
            each, tiles, lds, room = plan(act, 64, group * kv, kv, dim, 8192, accumulate)
            total = each * tiles * kv
            assert lds <= LDS and each <= room
            fit = UNITS * min(LDS // lds, 2)
            shares = (fit // 8 // tiles * 8 if tiles > 1 else fit) // kv * kv * tiles
            if 16 * shares >= 15 * fit:               # as many as fit leave few units idle: not more
                assert total <= fit, (kv, group, total, lds)
            assert 16 * total >= 15 * UNITS


def test_known_plans(plan):
    assert plan("f32", 64, 64, 8, 128, 7168, False)[0] * 8 == 512
    assert plan("bf16", 1, 32, 1, 128, 131072, True)[0] == 512
    assert plan("f32", 1, 32, 1, 128, 131072, False)[0] == 512
    assert plan("f32", 1, 32, 1, 128, 131072, True)[0] == 256          # 83200 bytes of LDS each
    assert plan("f32", 1, 32, 1, 128, 131072, True)[3] == 512
    assert plan("f32", 1, 8, 1, 256, 131072, True)[0] == 256
    assert plan("f32", 2, 8, 1, 128, 300, False)[0] == 6               # no more than there are steps
