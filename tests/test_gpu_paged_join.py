"""Keys that are split over workgroups: a value that is not finite reaches the rows that see it, however
small its weight and whatever the order of the parts."""
import itertools
import math

import pytest
import torch

import paper_2508_02401_amd as ckv
from tests.attn_ref import attend, check

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]
PAGE = 64


def _step(dt, d, n, add, low, total=None, bad=()):
    """`add` rows of 8 heads over the n tokens of one request. Keys low[0] .. low[1] lie 300 below the
    others in their logits; bad holds (key, column, value) of V, for KV head 1."""
    H, n_kv = 8, 2
    gen = torch.Generator().manual_seed(n + add)
    rand = lambda *shape: torch.randn(shape, generator=gen).to(dt).cuda()  # noqa: E731
    k, v, q = rand(n_kv, n, d), rand(n_kv, n, d), rand(add, H, d)
    q[:, :, 0], k[:, :, 0] = 10.0, 0.0
    k[:, low[0]:low[1], 0] = -30.0 * math.sqrt(d)
    kp, vp = (torch.zeros(-(-n // PAGE), n_kv, PAGE, d, dtype=dt, device="cuda") for _ in range(2))
    for key, c, x in bad:
        v[1, key, c] = x
    for x, pool in ((k, kp), (v, vp)):
        for p in range(pool.shape[0]):
            part = x[:, p * PAGE:(p + 1) * PAGE]
            pool[p, :, :part.shape[1]] = part
    ints = lambda xs: torch.tensor(xs, dtype=torch.int32, device="cuda")  # noqa: E731
    total = total or add
    desc = ckv.attn_desc(H, n_kv, d, dt)
    batch = ckv.paged_batch(ints([0, add]), ints([n]), ints([list(range(kp.shape[0]))]), total, add, n)
    qs = torch.zeros(total, H, d, dtype=dt, device="cuda")
    qs[:add] = q
    out = torch.full_like(qs, 7.0)
    ws = torch.empty(ckv.ckv_paged_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
    ckv.ckv_paged_attention(desc, ckv.paged_cache(kp, vp), batch, qs, out, ws)
    torch.cuda.synchronize()
    return q, k, v, out[:add]


# few rows, whose parts meet in one workgroup per row or in a few lanes; and the large row tiles.
# 100 keys are not split
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,add,total", [(6000, 1, None), (6000, 3, 800), (4000, 40, None), (4000, 40, 800),
                                         (100, 1, None)])
@pytest.mark.parametrize("side", ["first", "last"])
def test_values_of_little_weight_that_are_not_finite(dt, d, n, add, total, side):
    half = n // 2
    low = (0, half) if side == "first" else (half, n - add)
    key = low[0] + half // 3
    bad = [(key, 3, math.nan), (key + 1, 4, math.inf), (key + 5, 9, -math.inf)]
    q, k, v, plain = _step(dt, d, n, add, low, total)
    want, _, tol, _ = attend(q, k, v, torch.arange(n)[None] <= torch.arange(add)[:, None] + n - add)
    check(plain, want, tol, "finite values")
    _, _, _, out = _step(dt, d, n, add, low, total, bad)
    for h, c in itertools.product(range(8), range(d)):
        if h >= 4 and c in (3, 4, 9):
            assert not torch.isfinite(out[:, h, c]).any(), "head %d, column %d" % (h, c)
        else:
            assert torch.equal(out[:, h, c], plain[:, h, c]), "head %d, column %d" % (h, c)
