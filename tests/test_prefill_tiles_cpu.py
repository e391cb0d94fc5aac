"""The choice between small and large row tiles of packed prompts (csrc/ckv_plan.h compiled for the
host), against measured times of both."""
import ctypes
import itertools
import subprocess

import pytest

from paper_2508_02401_amd import build as B

# (fp32, (query heads, KV heads, head dim), prompts, us with large tiles, us with small ones)
MEASURED = [
    (False, (32, 8, 64), [1024], 26.0, 23.3), (False, (32, 8, 64), [2560], 57.6, 66.9),
    (False, (32, 8, 64), [320] * 4, 13.4, 19.9), (False, (16, 2, 64), [2048], 44.6, 31.6),
    (False, (16, 2, 64), [128] * 16, 11.5, 15.8), (False, (32, 8, 128), [512], 23.0, 16.7),
    (False, (32, 8, 128), [1280], 43.7, 50.9), (False, (32, 8, 128), [320] * 4, 19.3, 39.0),
    (False, (32, 8, 128), [320, 128, 32, 32], 18.0, 15.9), (False, (32, 8, 128), [2048], 65.9, 88.3),
    (True, (32, 8, 64), [2560], 352.6, 293.2), (True, (32, 8, 64), [4096], 603.1, 701.4),
    (True, (32, 8, 64), [1600, 640, 160, 160], 223.5, 169.0), (True, (32, 8, 64), [640] * 4, 94.6, 113.7),
    (True, (32, 8, 128), [1280], 322.7, 217.7), (True, (32, 8, 128), [2048], 514.8, 458.3),
    (True, (32, 8, 128), [320] * 4, 87.3, 114.7), (True, (32, 8, 128), [80] * 16, 27.0, 85.8),
    (True, (28, 4, 128), [2340], 590.2, 509.5), (True, (28, 4, 128), [585] * 4, 159.1, 225.4),
]


@pytest.fixture(scope="module")
def small(tmp_path_factory):
    d = tmp_path_factory.mktemp("tiles")
    src, lib = d / "shim.cpp", d / "shim.so"
    src.write_text(r"""
#include "ckv_plan.h"
extern "C" int small_tiles(int f32, int32_t d, int64_t G, int64_t n_kv, const int32_t* cu, int32_t n) {
  return ckv::prefill_small_tiles(f32 != 0, d, 256, 32, G, n_kv, cu, n);
}
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + B.CSRC, str(src),
                    "-o", str(lib)], check=True)
    so = ctypes.CDLL(str(lib))
    so.small_tiles.argtypes = [ctypes.c_int, ctypes.c_int32, ctypes.c_int64, ctypes.c_int64,
                               ctypes.POINTER(ctypes.c_int32), ctypes.c_int32]

    def choose(f32, shape, lens):
        H, n_kv, d = shape
        cu = list(itertools.accumulate([0] + lens))
        return bool(so.small_tiles(f32, d, H // n_kv, n_kv, (ctypes.c_int32 * len(cu))(*cu), len(lens)))
    return choose


@pytest.mark.parametrize("f32,shape,lens,large_us,small_us", MEASURED)
def test_the_faster_tiles(small, f32, shape, lens, large_us, small_us):
    assert small(f32, shape, lens) == (small_us < large_us)


def test_order_and_empty_prompts_do_not_count(small):
    for f32, shape, lens, _, _ in MEASURED:
        assert small(f32, shape, lens) == small(f32, shape, [0] + lens[::-1] + [0])
    # as long as prompts get
    assert not small(True, (128, 64, 128), [(1 << 29) - 1])
