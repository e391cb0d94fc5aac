"""Refusals of the prompt attention and the paged cache, which need no GPU: every bad argument
is answered with its status before anything is launched; and the bindings' own checks."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2508_02401_amd as ckv

# Fake device buffers: validation only looks at pointers, and every case below
# must fail before any HIP call.
_BUF = np.zeros(1 << 12, dtype=np.uint8)
_BASE = (_BUF.ctypes.data + 255) & ~255
INVALID, UNSUPPORTED, WORKSPACE = ckv.CKV_ERR_INVALID_ARG, ckv.CKV_ERR_UNSUPPORTED, ckv.CKV_ERR_WORKSPACE


def _fill(struct, vals, kw):
    for name, x in {**vals, **kw}.items():
        setattr(struct, name, x)
    return struct


def _desc(**kw):
    return _fill(ckv.attn_desc(8, 2, 64), {}, kw)


def _rows(**kw):
    return _fill(ckv.ckv_packed_attn(), dict(
        q=_BASE, k=_BASE + 16, v=_BASE + 32, out=_BASE + 48, q_stride_tok=512, q_stride_head=64,
        kv_stride_tok=128, kv_stride_head=64, out_stride_tok=512, out_stride_head=64,
        lse=_BASE + 64, lse_stride_head=100), kw)


def _cache(**kw):
    return _fill(ckv.ckv_paged_cache(), dict(
        k=_BASE, v=_BASE + 16, stride_page=2048, stride_head=1024, stride_tok=64, n_pages=10,
        page_size=16), kw)


def _batch(**kw):
    return _fill(ckv.ckv_paged_batch(), dict(
        cu_q=_BASE, kv_len=_BASE + 256, table=_BASE + 512, table_stride=8, table_width=8,
        num_seqs=3, total_q=20, max_q=10, max_kv=100), kw)


def _plan(**kw):
    return _fill(ckv.ckv_page_plan(), dict(
        cached=_BASE, add=_BASE + 64, num_seqs=3, page_size=16, table=_BASE + 128, table_stride=8,
        table_width=8, n_free=5, free_pages=_BASE + 256, free_head=_BASE + 320, cu_q=_BASE + 384,
        kv_len=_BASE + 448, slots=_BASE + 512, free_head_out=_BASE + 640, n_slots=30), kw)


BAD_DESC = [(dict(num_q_heads=7), INVALID), (dict(num_kv_heads=0), INVALID), (dict(num_q_heads=-8), INVALID),
            (dict(head_dim=96), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
            (dict(num_q_heads=130), UNSUPPORTED), (dict(num_q_heads=130, num_kv_heads=65), UNSUPPORTED),
            (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID)]
BAD_ROWS = [dict(q=None), dict(out=None), dict(q=_BASE + 8), dict(out=_BASE + 4), dict(q_stride_tok=508),
            dict(q_stride_tok=-512), dict(q_stride_head=32), dict(out_stride_tok=60), dict(out_stride_head=4),
            dict(out_stride_tok=0), dict(lse=_BASE + 2), dict(lse_stride_head=19), dict(lse_stride_head=-1)]


def _prefill(desc, a, cu, n=None):
    arr = None if cu is None else (ctypes.c_int32 * len(cu))(*cu)
    return ckv.load().ckv_prefill_attention(desc and ctypes.byref(desc), a and ctypes.byref(a), arr,
                                            len(cu) - 1 if n is None else n, None)


@pytest.mark.parametrize("bad,expect", BAD_DESC)
def test_descriptors(bad, expect):
    lib, d = ckv.load(), _desc(**bad)
    assert _prefill(d, _rows(), [0, 20]) == expect
    w = lib.ckv_paged_write(ctypes.byref(d), ctypes.byref(_cache()), _BASE, _BASE, 128, 64, _BASE, 3, None)
    assert w == expect
    b = _batch()
    assert lib.ckv_paged_workspace_bytes(ctypes.byref(d), ctypes.byref(b)) == 0
    assert _attention(d) == expect


@pytest.mark.parametrize("bad", BAD_ROWS + [
    dict(k=None), dict(v=None), dict(k=_BASE + 8), dict(v=_BASE + 1), dict(kv_stride_tok=60),
    dict(kv_stride_tok=-128), dict(kv_stride_head=12)])
def test_prefill_rows(bad):
    assert _prefill(_desc(), _rows(**bad), [0, 20]) == INVALID


def test_prefill_lengths():
    assert _prefill(None, _rows(), [0, 20]) == INVALID
    assert _prefill(_desc(), None, [0, 20]) == INVALID
    assert _prefill(_desc(), _rows(), None, 1) == INVALID
    assert _prefill(_desc(), _rows(), [0, 20], 0) == INVALID
    assert _prefill(_desc(), _rows(), [-1, 20]) == INVALID
    assert _prefill(_desc(), _rows(), [0, 20, 19]) == INVALID
    assert _prefill(_desc(), _rows(), [0, 2 ** 31 - 1]) == UNSUPPORTED
    # no token: nothing is looked at, nothing launched
    assert _prefill(_desc(), _rows(q=None), [4, 4, 4]) == ckv.CKV_OK


def _attention(desc=None, cache=None, batch=None, rows=None, ws=_BASE, n=1 << 40):
    desc, cache, batch, rows = desc or _desc(), cache or _cache(), batch or _batch(), rows or _rows()
    return ckv.load().ckv_paged_attention(ctypes.byref(desc), ctypes.byref(cache), ctypes.byref(batch),
                                          ctypes.byref(rows), ws, n, None)


BAD_CACHE = [dict(k=None), dict(v=None), dict(k=_BASE + 8), dict(n_pages=0), dict(page_size=0), dict(page_size=-4),
             dict(n_pages=1 << 20, page_size=1 << 11), dict(stride_page=60), dict(stride_tok=63),
             dict(stride_head=-64), dict(stride_tok=32), dict(stride_head=0)]


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_caches(bad):
    assert _attention(cache=_cache(**bad)) == INVALID
    c = _cache(**bad)
    assert ckv.load().ckv_paged_write(ctypes.byref(_desc()), ctypes.byref(c), _BASE, _BASE, 128, 64, _BASE, 3,
                                      None) == INVALID


@pytest.mark.parametrize("bad", BAD_ROWS)
def test_paged_rows(bad):
    assert _attention(rows=_rows(**bad)) == INVALID


@pytest.mark.parametrize("bad,expect", [
    (dict(cu_q=None), INVALID), (dict(kv_len=None), INVALID), (dict(table=None), INVALID),
    (dict(cu_q=_BASE + 2), INVALID), (dict(table=_BASE + 1), INVALID), (dict(table_width=0), INVALID),
    (dict(table_stride=7), INVALID), (dict(num_seqs=0), INVALID), (dict(total_q=-1), INVALID),
    (dict(max_q=-1), INVALID), (dict(max_kv=-1), INVALID), (dict(num_seqs=4097), UNSUPPORTED),
    (dict(total_q=1 << 29), UNSUPPORTED)])
def test_paged_batches(bad, expect):
    assert _attention(batch=_batch(**bad)) == expect


def test_paged_workspace_and_empty_steps():
    desc, batch = _desc(), _batch()
    need = ckv.ckv_paged_workspace_bytes(desc, batch)
    assert need > 0
    assert ckv.ckv_paged_workspace_bytes(desc, _batch(cu_q=None, kv_len=None, table=None)) == need
    assert _attention(ws=None) == WORKSPACE
    assert _attention(ws=_BASE + 8) == WORKSPACE
    assert _attention(n=need - 1) == WORKSPACE
    for none in (dict(total_q=0), dict(max_q=0)):
        assert _attention(batch=_batch(**none), ws=None, n=0) == ckv.CKV_OK
    # a larger step within every bound never needs less
    for more in (dict(total_q=40), dict(max_q=11), dict(max_kv=5000), dict(num_seqs=4)):
        assert ckv.ckv_paged_workspace_bytes(desc, _batch(**more)) >= need


@pytest.mark.parametrize("bad,expect", [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(slots=None), INVALID), (dict(k=_BASE + 8), INVALID),
    (dict(slots=_BASE + 1), INVALID), (dict(st=60), INVALID), (dict(st=-128), INVALID), (dict(sh=32), INVALID),
    (dict(n=-1), INVALID), (dict(n=1 << 31), INVALID), (dict(n=0, k=None, slots=None), ckv.CKV_OK)])
def test_writes(bad, expect):
    a = {**dict(k=_BASE, v=_BASE, st=128, sh=64, slots=_BASE, n=3), **bad}
    assert ckv.load().ckv_paged_write(ctypes.byref(_desc()), ctypes.byref(_cache()), a["k"], a["v"], a["st"], a["sh"],
                                      a["slots"], a["n"], None) == expect


@pytest.mark.parametrize("bad,expect", [
    (dict(cached=None), INVALID), (dict(add=None), INVALID), (dict(table=None), INVALID), (dict(cu_q=None), INVALID),
    (dict(kv_len=None), INVALID), (dict(slots=None), INVALID), (dict(free_head_out=None), INVALID),
    (dict(free_pages=None), INVALID), (dict(num_seqs=0), INVALID), (dict(num_seqs=4097), UNSUPPORTED),
    (dict(page_size=0), INVALID), (dict(table_width=0), INVALID), (dict(table_stride=7), INVALID),
    (dict(n_free=-1), INVALID), (dict(n_slots=-1), INVALID), (dict(cached=_BASE + 2), INVALID),
    # outputs over inputs or over each other, wholly or in part
    (dict(kv_len=_BASE), INVALID), (dict(cu_q=_BASE + 56), INVALID), (dict(free_head_out=_BASE + 320), INVALID),
    (dict(slots=_BASE + 244), INVALID), (dict(slots=_BASE + 396), INVALID), (dict(table=_BASE + 200), INVALID)])
def test_plans(bad, expect):
    p = _plan(**bad)
    assert ckv.load().ckv_paged_plan(ctypes.byref(p), None) == expect


def test_null_structs():
    lib = ckv.load()
    assert lib.ckv_paged_plan(None, None) == INVALID
    d, c, b, a = (ctypes.byref(x) for x in (_desc(), _cache(), _batch(), _rows()))
    assert lib.ckv_paged_attention(None, c, b, a, _BASE, 1 << 40, None) == INVALID
    assert lib.ckv_paged_attention(d, None, b, a, _BASE, 1 << 40, None) == INVALID
    assert lib.ckv_paged_attention(d, c, None, a, _BASE, 1 << 40, None) == INVALID
    assert lib.ckv_paged_attention(d, c, b, None, _BASE, 1 << 40, None) == INVALID
    assert lib.ckv_paged_write(d, None, _BASE, _BASE, 128, 64, _BASE, 3, None) == INVALID
    assert lib.ckv_paged_workspace_bytes(d, None) == 0


def test_bindings_refuse_what_they_cannot_pass():
    desc = ckv.attn_desc(4, 2, 64)
    q = torch.zeros(9, 4, 64, dtype=torch.bfloat16)
    k = torch.zeros(2, 9, 64, dtype=torch.bfloat16)
    lse = torch.zeros(4, 9)

    def prefill(q=q, k=k, v=None, cu=(0, 9), out=None, lse=lse):
        ckv.ckv_prefill_attention(desc, q, k, k if v is None else v, cu, torch.empty_like(q) if out is None else out, lse)

    for bad in (dict(q=q[:, :3]), dict(q=q.float()), dict(out=q.float()), dict(k=k[:1]), dict(v=k[:, :8]),
                dict(k=k[:, :8]), dict(cu=(0, 10)), dict(cu=(0,)), dict(lse=lse.double()), dict(lse=lse[:, :8]),
                dict(q=q.transpose(0, 2).contiguous().transpose(0, 2)), dict(k=k.half())):
        with pytest.raises(ValueError):
            prefill(**bad)
    with pytest.raises(ValueError, match="not on a GPU"):
        prefill()
    pool = torch.zeros(5, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ckv.paged_cache(pool, pool[:4])
    with pytest.raises(ValueError):
        ckv.paged_cache(pool.transpose(2, 3), pool.transpose(2, 3))
    cache, ints = ckv.paged_cache(pool, pool), torch.zeros(9, dtype=torch.int32)
    with pytest.raises(ValueError):  # another number of KV heads
        ckv.ckv_paged_write(ckv.attn_desc(4, 4, 64), cache, k, k, ints)
    with pytest.raises(ValueError):  # too few slots
        ckv.ckv_paged_write(desc, cache, k, k, ints[:8])
    with pytest.raises(ValueError):
        ckv.ckv_paged_write(desc, cache, k, k, ints.long())
    table = torch.zeros(3, 4, dtype=torch.int32)
    with pytest.raises(ValueError):
        ckv.paged_batch(ints[:3], ints[:3], table, 3, 1, 9)
    with pytest.raises(ValueError):
        ckv.paged_batch(ints[:4], ints[:3], table.t(), 3, 1, 9)
    batch = ckv.paged_batch(ints[:4], ints[:3], table, 10, 4, 9)
    with pytest.raises(ValueError, match="total_q"):
        ckv.ckv_paged_attention(desc, cache, batch, q, torch.empty_like(q), torch.zeros(10 ** 6))
    one = ints[:1]
    with pytest.raises(ValueError):
        ckv.ckv_paged_plan(ints[:3], ints[:2], table, 16, ints, one, ints[:4], ints[:3], ints, one)
    with pytest.raises(ValueError, match="not on a GPU"):
        ckv.ckv_paged_plan(ints[:3], ints[:3], table, 16, ints, one, ints[:4], ints[:3], ints, one)


def test_division_by_the_page_size(tmp_path):
    # csrc/ckv_plan.h compiled for the host: exact for every token number below 2^31, at the
    # edges of quotients and for every kind of page size
    import subprocess

    from paper_2508_02401_amd import build as B
    src, lib = tmp_path / "shim.cpp", tmp_path / "shim.so"
    src.write_text(r"""
#include "ckv_plan.h"
extern "C" int64_t wrong(int32_t size) {
  const ckv::PageDiv d = ckv::page_div(size);
  auto bad = [&](int64_t x) {
    return x >= 0 && x < (int64_t)1 << 31 && (int64_t)(((uint64_t)(uint32_t)x * d.mul) >> d.shift) != x / size;
  };
  int64_t n = 0;
  const int64_t most = ((int64_t)1 << 31) / size + 1, step = most < 100000 ? 1 : most / 99991;
  for (int64_t q = 0; q <= most; q += step)
    for (int64_t e = -1; e <= 1; ++e) n += bad(q * size + e);
  return n + bad(((int64_t)1 << 31) - 1);
}
""")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + B.CSRC, str(src),
                    "-o", str(lib)], check=True)
    so = ctypes.CDLL(str(lib))
    so.wrong.restype = ctypes.c_int64
    sizes = list(range(1, 300)) + [2 ** k + e for k in range(9, 31) for e in (-1, 0, 1)] + [2 ** 31 - 1]
    assert [s for s in sizes if so.wrong(s)] == []
