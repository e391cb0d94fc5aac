"""Prompt and paged attention on both sides of the rules that choose a kernel: prompts that fill the
chip with large row tiles, prompts in bands of position, and batches of many requests whose
keys are split or not, with a workspace that holds anything."""
import itertools
import math
import random

import pytest
import torch

import paper_2508_02401_amd as ckv
from tests.attn_ref import attend, check
from tests.test_gpu_paged import Step
from tests.test_gpu_prefill import _check, _inputs, _run

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _sums(xs):
    return list(itertools.accumulate([0] + list(xs)))


# 16 KV heads and one row tile or more of 256 rows per prompt: more than 256 tiles in all
LENS = [1, 0, 2, 31, 33, 63, 64, 65, 127, 129, 255, 256, 257, 300, 0, 513, 640, 705]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("H,d", [(16, 128), (48, 64)])
def test_large_row_tiles(dt, H, d):
    cu = _sums(LENS)
    q, k, v = _inputs(H + d, dt, H, 16, d, cu[-1])
    out, lse = _run(q, k, v, cu, 16)
    _check(q, k, v, cu, out, lse)


@pytest.mark.parametrize("dt", TYPES)
def test_large_row_tiles_with_values_that_are_not_finite(dt):
    cu = _sums(LENS)
    q, k, v = _inputs(5, dt, 16, 16, 128, cu[-1])
    for s, at, c, x in ((9, 0, 3, math.nan), (13, 77, 4, math.inf), (15, 200, 5, -math.inf),
                        (15, 300, 5, math.inf), (17, 704, 6, math.nan)):
        v[s - 2, cu[s] + at, c] = x
    out, lse = _run(q, k, v, cu, 16)
    _check(q, k, v, cu, out, lse)


@pytest.mark.parametrize("n", [2, 15, 16, 100, 240, 241, 500])
def test_prompts_in_bands(n):
    # every token once, whatever the number of prompts makes of the bands
    rng = random.Random(n)
    lens = [rng.choice([0, 1, rng.randint(1, 60), rng.randint(1, 3000 // n + 90)]) for _ in range(n)]
    cu = _sums(lens)
    q, k, v = _inputs(n, torch.bfloat16, 6, 2, 64, cu[-1])
    out, lse = _run(q, k, v, cu, 2)
    _check(q, k, v, cu, out, lse)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n", [63, 64, 65, 200])
def test_many_requests(dt, n):
    rng = random.Random(n)
    cached = [rng.choice([0, rng.randint(0, 80), rng.randint(0, 500)]) for _ in range(n)]
    add = [rng.choice([0, 1, 1, 1, 3, 20]) for _ in range(n)]
    cached[n // 2], cached[n - 1], add[n - 1], add[1] = 2000, 1300, 1, 70
    st = Step(n, dt, 8, 2, 64, 16, cached, add, spare=5)
    st.check(*st.run())


@pytest.mark.parametrize("dt", TYPES)
def test_both_kinds_of_requests_are_split(dt):
    st = Step(31, dt, 8, 2, 128, 32, [3000, 5000, 10, 1500], [100, 1, 90, 8])
    st.check(*st.run())


@pytest.mark.parametrize("fill", [0, 1, 127, 255])
def test_rows_of_no_request_stay_whatever_the_workspace_holds(fill):
    # rows before the first request's and behind the last one's, where keys are split; the same
    # workspace for a step whose rows lie elsewhere
    st = Step(32, torch.bfloat16, 8, 2, 64, 16, [2500, 40, 700], [2, 1, 45])
    want, want_lse = st.run()
    H, n_kv, d = st.shape
    desc = ckv.attn_desc(H, n_kv, d, torch.bfloat16)
    ints = lambda xs: torch.tensor(xs, dtype=torch.int32, device="cuda")  # noqa: E731
    ws = None
    for first, behind in ((3, 20), (0, 9), (11, 0)):
        n = first + 48 + behind
        q = torch.zeros(n, H, d, dtype=torch.bfloat16, device="cuda")
        q[first:first + 48] = st.q
        out, lse = torch.full_like(q, 7.0), torch.full((H, n), 7.0, device="cuda")
        batch = ckv.paged_batch(ints([first + x for x in _sums(st.add)]), ints(st.full), ints(st.table), n, 60, 4000)
        if ws is None:
            ws = torch.full((ckv.ckv_paged_workspace_bytes(desc, batch),), fill, dtype=torch.uint8, device="cuda")
        ckv.ckv_paged_attention(desc, ckv.paged_cache(st.k, st.v), batch, q, out, ws, lse=lse)
        torch.cuda.synchronize()
        rows = slice(first, first + 48)
        st.check(out[rows], lse[:, rows])
        assert (out[:first] == 7.0).all() and (out[first + 48:] == 7.0).all()
        assert (lse[:, :first] == 7.0).all() and (lse[:, first + 48:] == 7.0).all()


def test_shares_follow_the_lengths_within_one_graph():
    # one capture over lengths that are split and lengths that are not, replayed in turn
    H, n_kv, d, dt = 8, 2, 64, torch.float16
    steps = [Step(40 + i, dt, H, n_kv, d, 16, cached, [1, 40, 1], spare=9)
             for i, cached in enumerate(([2900, 10, 100], [5, 2800, 33], [60, 60, 60]))]
    desc = ckv.attn_desc(H, n_kv, d, dt)
    n_pages, width = max(s.k.shape[0] for s in steps), max(len(s.table[0]) for s in steps)
    kp, vp = (torch.zeros(n_pages, n_kv, 16, d, dtype=dt, device="cuda") for _ in range(2))
    table = torch.full((3, width), -1, dtype=torch.int32, device="cuda")
    kv = torch.zeros(3, dtype=torch.int32, device="cuda")
    cu = torch.tensor(_sums([1, 40, 1]), dtype=torch.int32, device="cuda")
    q, lse = torch.zeros(42, H, d, dtype=dt, device="cuda"), torch.zeros(H, 42, device="cuda")
    out = torch.zeros_like(q)
    batch = ckv.paged_batch(cu, kv, table, 42, 40, 3000)
    ws = torch.empty(ckv.ckv_paged_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
    cache, stream, graph = ckv.paged_cache(kp, vp), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            ckv.ckv_paged_attention(desc, cache, batch, q, out, ws, lse=lse)
    for i in (0, 1, 2, 0, 2, 1, 1):
        st = steps[i]
        kp[:st.k.shape[0]], vp[:st.k.shape[0]] = st.k, st.v
        table.fill_(-1)
        table[:, :len(st.table[0])] = torch.tensor(st.table, dtype=torch.int32, device="cuda")
        kv.copy_(torch.tensor(st.full, dtype=torch.int32)), q.copy_(st.q)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        st.check(out, lse)
        at = _sums(st.add)
        o, _, tol, _ = attend(*st.rows(1))
        check(out[at[1]:at[2]], o, tol, "step %d" % i)


def test_notes_of_rows_that_no_kernel_takes():
    # more rows than the bounds say: nobody writes their notes, and what the workspace held there
    # names parts of the large tiles' results, for which it has no room
    H, n_kv, d = 8, 2, 64
    st = Step(50, torch.bfloat16, H, n_kv, d, 16, [3000], [40])
    desc = ckv.attn_desc(H, n_kv, d, torch.bfloat16)
    ints = lambda xs: torch.tensor(xs, dtype=torch.int32, device="cuda")  # noqa: E731
    batch = ckv.paged_batch(ints([0, 40, 40]), ints([3040, 0]), ints(st.table * 2), 40, 1, 3040)
    n = ckv.ckv_paged_workspace_bytes(desc, batch)
    ws = torch.full((n // 8,), (2 << 32) + 0x80000000, dtype=torch.int64, device="cuda")
    out = torch.full((40, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    ckv.ckv_paged_attention(desc, ckv.paged_cache(st.k, st.v), batch, st.q, out, ws)
    torch.cuda.synchronize()
    assert (out == 7.0).all()


@pytest.mark.parametrize("add", [1, 60])
def test_pages_past_32_bits(add):
    # the request's pages lie behind the first 4 GiB of the pool, some before
    H, n_kv, d, page, n = 8, 2, 64, 64, 700
    gen = torch.Generator().manual_seed(add)
    n_pages = (5 << 30) // (n_kv * page * d * 2)
    pages = [n_pages - 1 - 3 * i if i % 3 else i for i in range(-(-n // page))]
    rand = lambda *shape: torch.randn(shape, generator=gen).to(torch.bfloat16).cuda()  # noqa: E731
    kp, vp = (torch.empty(n_pages, n_kv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v, q = rand(n_kv, n, d), rand(n_kv, n, d), rand(add, H, d)
    ints = lambda xs: torch.tensor(xs, dtype=torch.int32, device="cuda")  # noqa: E731
    desc, cache = ckv.attn_desc(H, n_kv, d), ckv.paged_cache(kp, vp)
    ckv.ckv_paged_write(desc, cache, k, v, ints([pages[j // page] * page + j % page for j in range(n)]))
    batch = ckv.paged_batch(ints([0, add]), ints([n]), ints([pages]), add, add, n)
    ws = torch.empty(ckv.ckv_paged_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(H, add, device="cuda")
    ckv.ckv_paged_attention(desc, cache, batch, q, out, ws, lse=lse)
    torch.cuda.synchronize()
    o, z, ot, zt = attend(q, k, v, torch.arange(n)[None] <= torch.arange(add)[:, None] + n - add)
    check(out, o, ot, "out")
    check(lse, z, zt, "lse")


@pytest.mark.parametrize("n,H", [(300, 2), (1100, 64)])
def test_rows_past_32_bits(n, H):
    # tokens of K and V so far apart that the last lies behind the first 4 GiB, on both sides
    # of the choice of tiles
    n_kv, d = H // 2, 64
    gap = (5 << 30) // 2 // n // 8 * 8
    q, k, v = _inputs(n, torch.bfloat16, H, n_kv, d, n)
    wide = torch.empty(n * gap + n_kv * d, dtype=torch.bfloat16, device="cuda")
    kw = wide.as_strided((n_kv, n, d), (d, gap, 1))
    vw = torch.empty_like(wide).as_strided((n_kv, n, d), (d, gap, 1))
    kw.copy_(k), vw.copy_(v)
    out, lse = _run(q, kw, vw, [0, n], n_kv)
    _check(q, k, v, [0, n], out, lse)
