"""How a paged request's keys are cut (csrc/ckv_plan.h compiled for the host), up to the longest that
ckv_paged_attention takes."""
import ctypes
import random
import subprocess

import pytest

from paper_2508_02401_amd import build as B

LONGEST = 0x7FFFF000  # CKV_MAX_PAGED_KV
UNSPLIT = 0x7FFFFF80  # the share of a batch that is not split


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    d = tmp_path_factory.mktemp("cut")
    src, lib = d / "shim.cpp", d / "shim.so"
    src.write_text(r"""
#include "ckv_plan.h"
extern "C" {
int32_t chunks(int32_t n, int32_t chunk) { return ckv::paged_chunks(n, chunk); }
int32_t chunk_end(int32_t n, int32_t chunk, int32_t c) { return ckv::paged_chunk_end(n, chunk, c); }
}
""")
    subprocess.run(["g++", "-std=c++17", "-O2", "-ftrapv", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + B.CSRC,
                    str(src), "-o", str(lib)], check=True)
    return ctypes.CDLL(str(lib))


def _share(work, parts, least, unit):
    """Keys per workgroup, as the kernels work it out."""
    return min(max(-(-work // (parts * unit)) * unit, least), UNSPLIT)


def _cases():
    rng = random.Random(1)
    lens = [0, 1, 127, 128, 129, 1023, 1024, 1025, 10 ** 6, 2 ** 30, LONGEST - 129, LONGEST - 1, LONGEST]
    lens += [rng.randrange(1, LONGEST) for _ in range(200)]
    for n in lens:
        for unit, least, targets in ((128, 128, (256, 512, 768, 1536)), (64, 1024, (256, 255, 129, 128))):
            for parts in targets:
                for n_kv in (1, 3, 64):
                    yield n, _share(n * n_kv, parts, least, unit)
                    yield n, _share((n + rng.randrange(LONGEST)) * n_kv, parts, least, unit)
        yield n, UNSPLIT


def test_every_key_lies_in_one_chunk(cut):
    # one request of 2^31 - 4096 keys gets shares of 4194304, and their sum passes 2^31
    assert (LONGEST, 4194304) in set(_cases())
    for n, chunk in _cases():
        count = cut.chunks(n, chunk)
        assert count == max(1, -(-n // chunk)), (n, chunk)
        for c in {0, count // 2, count - 1}:
            assert cut.chunk_end(n, chunk, c) == min(n, (c + 1) * chunk), (n, chunk, c)
