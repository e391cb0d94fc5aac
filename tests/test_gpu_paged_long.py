"""Paged attention where one request's length is the longest that the bounds can name."""
import pytest
import torch

import paper_2508_02401_amd as ckv
from tests.attn_ref import attend, check

pytestmark = pytest.mark.gpu

LONGEST = 0x7FFFF000  # CKV_MAX_PAGED_KV


@pytest.mark.parametrize("page", [1, 16])
@pytest.mark.parametrize("add", [1, 40])
def test_a_length_past_the_table(add, page):
    # 2^31 - 4096 tokens of which the table has 320: those are what its rows see, and the requests
    # before and behind it come out as they are
    dt, H, n_kv, d, have = torch.bfloat16, 4, 1, 64, 320
    gen = torch.Generator().manual_seed(add + page)
    rand = lambda *shape: torch.randn(shape, generator=gen).to(dt).cuda()  # noqa: E731
    ints = lambda xs: torch.tensor(xs, dtype=torch.int32, device="cuda")  # noqa: E731
    width = have // page
    kp, vp = (rand(3 * width, n_kv, page, d) for _ in range(2))
    table = torch.randperm(3 * width, generator=gen).view(3, width)
    lens, rows = [have, LONGEST, have - 9], [0, add, 2 * add, 3 * add]
    q = rand(3 * add, H, d)
    desc = ckv.attn_desc(H, n_kv, d, dt)
    batch = ckv.paged_batch(ints(rows), ints(lens), ints(table.tolist()), 3 * add, add, LONGEST)
    ws = torch.empty(ckv.ckv_paged_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.full((H, 3 * add), 7.0, device="cuda")
    ckv.ckv_paged_attention(desc, ckv.paged_cache(kp, vp), batch, q, out, ws, lse=lse)
    torch.cuda.synchronize()
    for s in range(3):
        k, v = (x[table[s].cuda()].transpose(0, 1).flatten(1, 2) for x in (kp, vp))
        seen = torch.arange(have)[None] <= torch.arange(add)[:, None] + lens[s] - add
        at = slice(rows[s], rows[s + 1])
        o, z, ot, zt = attend(q[at], k, v, seen)
        check(out[at], o, ot, "out of request %d" % s)
        check(lse[:, at], z, zt, "lse of request %d" % s)
