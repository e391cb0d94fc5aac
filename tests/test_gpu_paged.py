"""The paged cache: ckv_paged_plan and ckv_paged_write exactly, ckv_paged_attention against plain
64-bit attention, and a run of all of them with the prompt's attention and its compression."""
import itertools
import math
import random

import pytest
import torch

import paper_2508_02401_amd as ckv
from tests.attn_ref import attend, check

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _sums(xs):
    return list(itertools.accumulate([0] + list(xs)))


def _ints(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def _rand(gen, dt, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float32).to(dt).cuda()


def plan_reference(cached, add, table, page, free, head, n_slots):
    """The documented result, number after number."""
    table = [list(r) for r in table]
    width = len(table[0])
    cu = _sums(max(x, 0) for x in add)
    slots, start = [], head
    for s, (c, a) in enumerate(zip(cached, add)):
        c, a = max(c, 0), max(a, 0)
        for p in range(min(-(-c // page), width), min(-(-(c + a) // page), width)):
            table[s][p] = free[head] if head < len(free) else -1
            head += 1
        for pos in range(c, c + a):
            p = pos // page
            ok = p < width and table[s][p] >= 0
            slots.append(table[s][p] * page + pos % page if ok else -1)
    slots = (slots + [-1] * n_slots)[:n_slots]
    return table, cu, [max(c, 0) + max(a, 0) for c, a in zip(cached, add)], slots, head


def run_plan(cached, add, table, page, free, head, n_slots):
    t = _ints(table)
    cu, kv = _ints([9] * (len(add) + 1)), _ints([9] * len(add))
    slots, out = torch.full((n_slots,), 9, dtype=torch.int32, device="cuda"), _ints([9])
    ckv.ckv_paged_plan(_ints(cached), _ints(add), t, page, _ints(free),
                       None if head is None else _ints([head]), cu, kv, slots, out)
    torch.cuda.synchronize()
    return t.tolist(), cu.tolist(), kv.tolist(), slots.tolist(), int(out)


def make_tables(rng, cached, page, width, spare):
    """Block tables of shuffled pages that hold the cached tokens, and a shuffled free list."""
    need = sum(-(-c // page) for c in cached)
    pages = list(range(need + spare))
    rng.shuffle(pages)
    table, at = [], 0
    for c in cached:
        n = -(-c // page)
        table.append(pages[at:at + n] + [-1] * (width - n))
        at += n
    return table, pages[at:]


@pytest.mark.parametrize("n", [1, 3, 64, 255, 256, 257, 1000, 4096])
@pytest.mark.parametrize("page", [1, 16, 24])
def test_plan(n, page):
    rng = random.Random(n * 100 + page)
    most = 300 if n <= 64 else 20
    cached = [rng.choice([0, 1, page, page - 1, rng.randint(0, most)]) for _ in range(n)]
    add = [rng.choice([0, 1, 1, page, rng.randint(0, most)]) for _ in range(n)]
    width = 2 * most // page + 4
    table, free = make_tables(rng, cached, page, width, sum(add) // page + n + 5)
    for n_slots in (sum(add), sum(add) + 77, max(0, sum(add) - 1)):
        want = plan_reference(cached, add, table, page, free, 2, n_slots)
        assert run_plan(cached, add, table, page, free, 2, n_slots) == want


def test_plan_where_pages_are_missing():
    rng = random.Random(5)
    cached, add, page = [10, 0, 33, 7, 40], [30, 5, 0, 200, 9], 16
    # the free list ends, the table is too narrow, a page that was taken away, negative lengths
    for width, spare in ((20, 4), (20, 0), (4, 30)):
        have = [min(c, width * page) for c in cached]
        table, free = make_tables(rng, have, page, width, spare)
        table[0][0] = -1
        for head in (0, None):
            want = plan_reference(cached, add, table, page, free, 0, 260)
            assert run_plan(cached, add, table, page, free, head, 260) == want
    table, free = make_tables(rng, [0, 5], page, 8, 9)
    want = plan_reference([-4, 5], [3, -2], table, page, free, 1, 8)
    assert run_plan([-4, 5], [3, -2], table, page, free, 1, 8) == want


def test_plan_of_long_prompts():
    # slots and new pages over many workgroups
    rng = random.Random(6)
    cached, add, page = [100001, 0, 17], [1, 70000, 30011], 64
    width = 2000
    table, free = make_tables(rng, cached, page, width, 2000)
    want = plan_reference(cached, add, table, page, free, 3, 100100)
    assert run_plan(cached, add, table, page, free, 3, 100100) == want


def _pool(gen, dt, n_pages, n_kv, page, d, slot_major):
    if slot_major:
        return tuple(_rand(gen, dt, n_pages, page, n_kv, d).transpose(1, 2) for _ in range(2))
    return tuple(_rand(gen, dt, n_pages, n_kv, page, d) for _ in range(2))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,page,slot_major,head_major", [
    (1, 16, False, False), (37, 24, True, False), (500, 16, False, True), (129, 1, True, True)])
def test_write(dt, d, n, page, slot_major, head_major):
    gen, rng = torch.Generator().manual_seed(n + d), random.Random(n)
    n_kv, n_pages = 3, -(-n // page) + 7
    kp, vp = _pool(gen, dt, n_pages, n_kv, page, d, slot_major)
    k, v = (_rand(gen, dt, n_kv, n, d) if head_major else _rand(gen, dt, n, n_kv, d).transpose(0, 1)
            for _ in range(2))
    slots = rng.sample(range(n_pages * page), n)
    for i in range(0, n, 5):  # left out: no slot, and slots past the pool
        slots[i] = rng.choice([-1, -7, n_pages * page, n_pages * page + 3, 2 ** 31 - 1])
    want_k, want_v = kp.clone(), vp.clone()
    for r, s in enumerate(slots):
        if 0 <= s < n_pages * page:
            want_k[s // page, :, s % page], want_v[s // page, :, s % page] = k[:, r], v[:, r]
    desc = ckv.attn_desc(n_kv, n_kv, d, dt)
    ckv.ckv_paged_write(desc, ckv.paged_cache(kp, vp), k, v, _ints(slots))
    torch.cuda.synchronize()
    assert torch.equal(kp, want_k) and torch.equal(vp, want_v)


class Step:
    """A batch over a paged cache, with everything that a row does not see set to NaN."""

    def __init__(self, seed, dt, H, n_kv, d, page, cached, add, slot_major=False, poison=True, spare=3):
        gen, rng = torch.Generator().manual_seed(seed), random.Random(seed)
        full = [c + a for c, a in zip(cached, add)]
        self.shape, self.page, self.add, self.full = (H, n_kv, d), page, add, full
        width = max(max(-(-x // page) for x in full), 1) + 2
        self.table, _ = make_tables(rng, full, page, width, spare)
        n_pages = sum(-(-x // page) for x in full) + spare
        self.k, self.v = _pool(gen, dt, n_pages, n_kv, page, d, slot_major)
        self.q = _rand(gen, dt, max(sum(add), 1), H, d)
        if poison:
            used = torch.zeros(n_pages, page, dtype=torch.bool)
            for row, x in zip(self.table, full):
                for j in range(x):
                    used[row[j // page], j % page] = True
            hole = (~used).cuda()[:, None, :, None].expand(self.k.shape)
            self.k.masked_fill_(hole, math.nan), self.v.masked_fill_(hole, math.inf)

    def run(self, total=None, max_q=None, max_kv=None, scale=0.0, lse=True, ws=None):
        H, n_kv, d = self.shape
        desc = ckv.attn_desc(H, n_kv, d, self.q.dtype, scale)
        total = sum(self.add) if total is None else total
        batch = ckv.paged_batch(_ints(_sums(self.add)), _ints(self.full), _ints(self.table), total,
                                max(self.add) if max_q is None else max_q,
                                max(self.full) if max_kv is None else max_kv)
        out = torch.full(self.q.shape, 7.0, dtype=self.q.dtype, device="cuda")
        z = torch.full((H, self.q.shape[0]), 7.0, device="cuda") if lse else None
        n = ckv.ckv_paged_workspace_bytes(desc, batch)
        assert n > 0
        if ws is None:
            # scratch starts as it may: NaN
            ws = torch.full((n // 4 + 4,), math.nan, device="cuda")
        ckv.ckv_paged_attention(desc, ckv.paged_cache(self.k, self.v), batch, self.q, out, ws, lse=z)
        torch.cuda.synchronize()
        return out, z

    def rows(self, s):
        """Request s's queries, its keys and values in order, and which of them a row sees."""
        a = _sums(self.add)
        T, n = self.add[s], self.full[s]
        n_pages = self.k.shape[0]
        pages = [self.table[s][j // self.page] if j // self.page < len(self.table[s]) else -1 for j in range(n)]
        there = torch.tensor([0 <= p < n_pages for p in pages], dtype=torch.bool)
        at = torch.tensor([p if 0 <= p < n_pages else 0 for p in pages], dtype=torch.long).cuda()
        slot = (torch.arange(n) % self.page).cuda()
        k, v = (x[at, :, slot].transpose(0, 1) if n else x[:0, :, 0].transpose(0, 1) for x in (self.k, self.v))
        seen = torch.arange(n)[None] <= torch.arange(T)[:, None] + (n - T)
        seen = seen & there[None]
        hidden = ~seen.any(0) if T else torch.ones(n, dtype=torch.bool)
        k, v = k.clone(), v.clone()
        k[:, hidden], v[:, hidden] = 0, 0  # whatever they hold, nobody sees them
        return self.q[a[s]:a[s + 1]], k, v, seen

    def check(self, out, lse, scale=0.0):
        cu = _sums(self.add)
        for s in range(len(self.add)):
            if self.add[s] == 0:
                continue
            q, k, v, seen = self.rows(s)
            o, z, ot, zt = attend(q, k, v, seen, scale)
            check(out[cu[s]:cu[s + 1]], o, ot, "out of request %d" % s)
            if lse is not None:
                check(lse[:, cu[s]:cu[s + 1]], z, zt, "lse of request %d" % s)
        assert (out[cu[-1]:] == 7.0).all()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("H,n_kv,d,page", [(8, 2, 64, 16), (28, 4, 128, 24), (4, 4, 128, 64), (32, 2, 64, 1),
                                           (3, 1, 128, 7)])
def test_single_tokens(dt, H, n_kv, d, page):
    cached = [0, 1, 30, 31, 32, 62, 63, 64, 100, 127, 128, 700, 1500]
    st = Step(H + d + page, dt, H, n_kv, d, page, cached, [1] * len(cached))
    st.check(*st.run())


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("H,n_kv,d,page", [(8, 2, 64, 16), (28, 4, 128, 24), (5, 5, 128, 48)])
def test_chunks_and_mixes(dt, H, n_kv, d, page):
    cached = [0, 500, 33, 1000, 64, 0, 7, 90]
    add = [90, 1, 0, 300, 17, 1, 5, 64]
    st = Step(H * d + page, dt, H, n_kv, d, page, cached, add, slot_major=True)
    st.check(*st.run())
    # the same within wider bounds, as a captured step has them: to the bit where the same
    # kernels run, within the same tolerances otherwise
    st.q = torch.cat([st.q, st.q[:50]])
    st.check(*st.run(total=sum(add) + 50, max_q=400, max_kv=4000))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_long_cache_is_split(dt):
    st = Step(3, dt, 8, 1, 128, 32, [9000], [1])
    st.check(*st.run())
    st = Step(4, dt, 8, 1, 64, 16, [5000, 9], [40, 3])
    st.check(*st.run())


@pytest.mark.parametrize("dt", TYPES)
def test_values_that_are_not_finite(dt):
    # among the new tokens (seen by some of the rows), and among the old ones (seen by all)
    for add in ([6, 1, 3], [40, 1, 80]):
        st = Step(11, dt, 4, 2, 64, 16, [50, 3, 200], add)
        for s, j, g, c, x in ((0, 52, 0, 4, math.inf), (2, 201, 1, 7, math.nan), (2, 17, 0, 9, -math.inf),
                              (0, 53, 0, 4, -math.inf)):
            st.v[st.table[s][j // 16], g, j % 16, c] = x
        st.check(*st.run())


def test_rows_that_see_nothing():
    # fewer tokens than rows, none at all, and pages that are not there
    for add in ([4, 3, 2, 1, 2], [40, 70, 33, 1, 50]):
        st = Step(12, torch.bfloat16, 8, 2, 64, 16, [60, 20, 0, 300, 0], add)
        st.full[0], st.full[2], st.full[4] = 2, 0, 1
        st.table[1] = [-1] * len(st.table[1])
        n_pages = st.k.shape[0]
        st.table[3] = [n_pages, -5, 2 ** 31 - 1, -2 ** 31] + st.table[3][4:]
        out, lse = st.run()
        st.check(out, lse)
        cu = _sums(add)
        assert (out[cu[1]:cu[2]] == 0).all() and (lse[:, cu[1]:cu[2]] == -math.inf).all()
        assert (out[cu[2]:cu[3]] == 0).all()


def test_numbers_out_of_bounds_stay_inside():
    # device arrays that break the bounds: any result, but nothing outside the arrays, and the
    # requests that keep to them unharmed
    st = Step(13, torch.bfloat16, 8, 2, 64, 16, [60, 20, 100], [1, 1, 1])
    want, _ = st.run()
    H, n_kv, d = st.shape
    desc = ckv.attn_desc(H, n_kv, d, torch.bfloat16)
    out = torch.full((3, H, d), 7.0, dtype=torch.bfloat16, device="cuda")
    for cu, kv in (([0, 1, 2, 3], [61, 2 ** 31 - 1, 101]), ([0, 1, 2, 3], [61, -9, 101]),
                   ([0, 1, 1, 2 ** 31 - 1], [61, 21, 101]), ([-5, 1, 2, 3], [61, 21, 101])):
        batch = ckv.paged_batch(_ints(cu), _ints(kv), _ints(st.table), 3, 1, 101)
        ws = torch.zeros(ckv.ckv_paged_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
        ckv.ckv_paged_attention(desc, ckv.paged_cache(st.k, st.v), batch, st.q, out, ws)
        torch.cuda.synchronize()
        if cu == [0, 1, 2, 3]:
            assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2])


def test_same_results_every_time():
    st = Step(14, torch.bfloat16, 28, 4, 128, 16, [3000, 70, 1200, 5], [1, 60, 4, 1])
    want, want_lse = st.run()
    for _ in range(5):
        out, lse = st.run()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_a_graph_serves_every_step_within_its_bounds():
    # one capture, replayed over steps of growing lengths, tables planned inside the graph
    H, n_kv, d, page, dt = 8, 2, 128, 16, torch.bfloat16
    desc = ckv.attn_desc(H, n_kv, d, dt)
    gen = torch.Generator().manual_seed(15)
    n, width, steps = 3, 8, 6
    cached, add = _ints([0, 37, 15]), _ints([1, 1, 1])
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    table[1, :3], table[2, 0] = _ints([4, 9, 2]), 7
    free = _ints([1, 3, 0, 5, 6, 8, 10, 11])
    head, head_out = _ints([0]), _ints([0])
    cu, kv, slots = _ints([0] * (n + 1)), _ints([0] * n), _ints([0] * n)
    kp, vp = _pool(gen, dt, 12, n_kv, page, d, False)
    q, out, lse = torch.zeros(n, H, d, dtype=dt, device="cuda"), torch.zeros(n, H, d, dtype=dt, device="cuda"), torch.zeros(H, n, device="cuda")
    kn, vn = torch.zeros(2, n, n_kv, d, dtype=dt, device="cuda").unbind()
    batch = ckv.paged_batch(cu, kv, table, n, 1, 100)
    ws = torch.empty(ckv.ckv_paged_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
    cache = ckv.paged_cache(kp, vp)

    def step():
        ckv.ckv_paged_plan(cached, add, table, page, free, head, cu, kv, slots, head_out)
        ckv.ckv_paged_write(desc, cache, kn.transpose(0, 1), vn.transpose(0, 1), slots)
        ckv.ckv_paged_attention(desc, cache, batch, q, out, ws, lse=lse)

    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    before = kp.clone(), vp.clone(), table.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
    kp.copy_(before[0]), vp.copy_(before[1]), table.copy_(before[2])
    tokens = [[], [], []]
    for s in range(n):
        for j in range(int(cached[s])):
            p = int(table[s, j // page])
            tokens[s].append((kp[p, :, j % page].clone(), vp[p, :, j % page].clone()))
    for i in range(steps):
        q.copy_(_rand(gen, dt, n, H, d)), kn.copy_(_rand(gen, dt, n, n_kv, d)), vn.copy_(_rand(gen, dt, n, n_kv, d))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for s in range(n):
            tokens[s].append((kn[s].clone(), vn[s].clone()))
            k, v = (torch.stack([t[x] for t in tokens[s]], 1) for x in range(2))
            o, z, ot, zt = attend(q[s:s + 1], k, v, torch.ones(1, k.shape[1], dtype=torch.bool))
            check(out[s:s + 1], o, ot, "step %d, request %d" % (i, s))
            check(lse[:, s:s + 1], z, zt, "step %d, request %d" % (i, s))
        cached.copy_(kv), head.copy_(head_out)
    assert cached.tolist() == [steps, 37 + steps, 15 + steps]


def test_two_streams():
    a = Step(16, torch.bfloat16, 8, 2, 128, 16, [3000], [1])
    b = Step(17, torch.bfloat16, 8, 2, 128, 16, [900, 10], [70, 2])
    want = a.run()[0], b.run()[0]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[], []]
    for _ in range(4):
        for i, (st, x) in enumerate(zip(streams, (a, b))):
            with torch.cuda.stream(st):
                H, n_kv, d = x.shape
                desc = ckv.attn_desc(H, n_kv, d, x.q.dtype)
                batch = ckv.paged_batch(_ints(_sums(x.add)), _ints(x.full), _ints(x.table), sum(x.add), max(x.add), max(x.full))
                ws = torch.empty(ckv.ckv_paged_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
                out = torch.empty_like(x.q)
                ckv.ckv_paged_attention(desc, ckv.paged_cache(x.k, x.v), batch, x.q, out, ws)
                outs[i].append((out, ws, batch))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o[0], want[i]) for o in outs[i])


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_prompt_to_compressed_cache_to_decoding(dt):
    """As a server runs them: the prompts' attention, their compression with its log-sum-exp, the
    compact rows into pages, then chunks and single tokens over them."""
    H, n_kv, d, w, page, lens, budget = 8, 2, 128, 16, 16, [600, 250], [90, 61]
    gen = torch.Generator().manual_seed(18)
    cu = _sums(lens)
    desc, layer = ckv.attn_desc(H, n_kv, d, dt), ckv.layer_desc(H, n_kv, d, w, dt)
    q, kn, vn = (_rand(gen, dt, cu[-1], h, d) for h in (H, n_kv, n_kv))
    k, v = kn.transpose(0, 1), vn.transpose(0, 1)
    out, lse = torch.empty_like(q), torch.empty(H, cu[-1], device="cuda")
    ckv.ckv_prefill_attention(desc, q, k, v, cu, out, lse=lse)
    seqs = [ckv.alloc_outputs(layer, ckv.Seq(q[b - w:b].transpose(0, 1), k[:, a:b], v[:, a:b], n, lse=lse[:, b - w:b]))
            for a, b, n in zip(cu, cu[1:], budget)]
    ckv.ckv_compress_layer(layer, [0, 1, 1, 0, 1, 0, 0, 1], seqs, ckv.alloc_workspace(layer, seqs, "cuda"))
    kp, vp = _pool(gen, dt, 40, n_kv, page, d, False)
    cache = ckv.paged_cache(kp, vp)
    table = torch.full((2, 16), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(40, generator=gen).to(torch.int32).cuda()
    cached, head = _ints([0, 0]), _ints([0])
    kv, cu_q, head_out = _ints([0, 0]), _ints([0, 0, 0]), _ints([0])
    have = [(s.k_out.clone(), s.v_out.clone()) for s in seqs]
    # the compact rows, request after request
    slots = torch.empty(sum(budget), dtype=torch.int32, device="cuda")
    ckv.ckv_paged_plan(cached, _ints(budget), table, page, free, head, cu_q, kv, slots, head_out)
    for s, a in zip(seqs, _sums(budget)):
        ckv.ckv_paged_write(desc, cache, s.k_out, s.v_out, slots[a:a + s.k_out.shape[1]])
    for add in ([1, 1], [20, 1], [3, 40], [1, 1]):
        cached.copy_(kv), head.copy_(head_out)
        n = sum(add)
        slots = torch.empty(n + 3, dtype=torch.int32, device="cuda")
        ckv.ckv_paged_plan(cached, _ints(add), table, page, free, head, cu_q, kv, slots, head_out)
        q, kn, vn = (_rand(gen, dt, n, h, d) for h in (H, n_kv, n_kv))
        ckv.ckv_paged_write(desc, cache, kn.transpose(0, 1), vn.transpose(0, 1), slots)
        batch = ckv.paged_batch(cu_q, kv, table, n, max(add), 256)
        ws = torch.empty(ckv.ckv_paged_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
        out, lse = torch.empty_like(q), torch.empty(H, n, device="cuda")
        ckv.ckv_paged_attention(desc, cache, batch, q, out, ws, lse=lse)
        torch.cuda.synchronize()
        at = _sums(add)
        for s in range(2):
            new = slice(at[s], at[s + 1])
            have[s] = tuple(torch.cat([x, y[new].transpose(0, 1)], 1) for x, y in zip(have[s], (kn, vn)))
            n_all, T = have[s][0].shape[1], add[s]
            seen = torch.arange(n_all)[None] <= torch.arange(T)[:, None] + n_all - T
            o, z, ot, zt = attend(q[new], have[s][0], have[s][1], seen)
            check(out[new], o, ot, "request %d" % s)
            check(lse[:, new], z, zt, "request %d" % s)
