"""How exact the weights of 16-bit types are: single and drafted tokens over a paged cache come out as
those over a contiguous one (ckv_decode_attention), to the rounding of their outputs."""
import math

import pytest
import torch

import paper_2508_02401_amd as ckv
from tests.attn_ref import attend

pytestmark = pytest.mark.gpu

PAGE = 16


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,add", [(40, 1), (100, 4), (1500, 1), (900, 8)])
def test_rounded_to_two_parts(dt, d, n, add):
    H, n_kv = 8, 2
    gen = torch.Generator().manual_seed(n + d)
    rand = lambda *shape: torch.randn(shape, generator=gen).to(dt).cuda()  # noqa: E731
    ints = lambda xs: torch.tensor(xs, dtype=torch.int32, device="cuda")  # noqa: E731
    width = -(-n // PAGE)
    kp, vp, q = rand(width, n_kv, PAGE, d), rand(width, n_kv, PAGE, d), rand(add, H, d)
    desc = ckv.attn_desc(H, n_kv, d, dt)
    batch = ckv.paged_batch(ints([0, add]), ints([n]), ints([list(range(width))]), add, add, n)
    ws = torch.empty(ckv.ckv_paged_workspace_bytes(desc, batch), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    ckv.ckv_paged_attention(desc, ckv.paged_cache(kp, vp), batch, q, out, ws)
    torch.cuda.synchronize()
    k, v = (x.transpose(0, 1).flatten(1, 2)[:, :n] for x in (kp, vp))
    seen = torch.arange(n)[None] <= torch.arange(add)[:, None] + n - add
    want, _, _, _ = attend(q, k, v, seen)
    # A = sum w |v| bounds an output. Each weight is off by its low part's rounding, half a step
    # relative to a remainder that is at most half a step of the weight: half^2 (f16 low parts
    # are multiples of 2^-24 after being raised by 2^8: off by at most 2^-33 of the largest
    # weight besides). The logits' d + 4 roundings of 2^-24 of S = sum |q k| scale count as
    # relative errors of the weights, twice (product and normaliser), exp2 4 more, and n terms
    # are summed twice in fp32. Last, half a step of the output
    half, u = torch.finfo(dt).eps / 2, 2.0 ** -24
    for h in range(H):
        qh, kh, vh = q[:, h].cpu().double(), k[h // 4].cpu().double(), v[h // 4].cpu().double()
        z = (qh @ kh.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
        w = torch.softmax(z, 1)
        size = (qh.abs() @ kh.abs().T / math.sqrt(d)).amax(1, keepdim=True)
        rel = half * half + 2 * ((d + 4) * u * size + 4 * u) + 2 * n * u
        tol = rel * (w @ vh.abs()) + half * want[:, h].abs()
        if dt == torch.float16:
            tol = tol + n * 2.0 ** -33 * w.amax(1, keepdim=True) * vh.abs().amax()
        over = ((out[:, h].cpu().double() - want[:, h]).abs() / tol).max()
        assert over <= 1.0, "head %d: %.2f times its tolerance" % (h, float(over))
