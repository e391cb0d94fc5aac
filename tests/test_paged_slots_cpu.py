"""Where the parts of split requests lie in the workspace (csrc/ckv_plan.h compiled for the host)."""
import ctypes
import subprocess

import pytest

import paper_2508_02401_amd as ckv
from paper_2508_02401_amd import build as B


@pytest.mark.parametrize("d", [64, 128])
def test_slots_are_whole_16_bytes(tmp_path, d):
    src, lib = tmp_path / "shim.cpp", tmp_path / "shim.so"
    src.write_text('#include "ckv_plan.h"\n'
                   'extern "C" int64_t words(int32_t rows, int32_t d) { return ckv::partial_words(rows, d); }\n')
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + B.CSRC, str(src),
                    "-o", str(lib)], check=True)
    so = ctypes.CDLL(str(lib))
    so.words.restype = ctypes.c_int64
    for rows in range(1, 257):
        assert so.words(rows, d) % 4 == 0 and rows * (d + 2) <= so.words(rows, d) < rows * (d + 2) + 4


@pytest.mark.parametrize("H,n_kv", [(28, 4), (3, 1), (5, 5), (8, 2)])
@pytest.mark.parametrize("max_q", [1, 3, 60])
def test_workspace_parts_are_whole_16_bytes(H, n_kv, max_q):
    # slots of few rows, slots of the large tiles, notes of 8 bytes per row, 256 bytes
    b = ckv.ckv_paged_batch()
    b.num_seqs, b.total_q, b.max_q, b.max_kv = 3, 60, max_q, 9000
    desc = ckv.attn_desc(H, n_kv, 128)
    parts = ckv.ckv_paged_workspace_bytes(desc, b) - 60 * H * 8 - 256
    few = min(max_q * H // n_kv, 32)
    many = 256 * (256 * 130 * 4) if max_q * H // n_kv > 32 else 0
    slot = (few * 130 + 3) // 4 * 16
    assert parts - many > 0 and (parts - many) % slot == 0
