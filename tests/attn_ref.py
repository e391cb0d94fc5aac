"""Plain 64-bit attention of rows that see the first keys of a request, and how far a
kernel's fp32 arithmetic may be from it."""
from __future__ import annotations

import math

import torch


def attend(q, k, v, seen, scale=0.0):
    """q [T, H, d], k, v [n_kv, n, d], seen [T, n] bool (which keys a row sees). Returns out
    [T, H, d], lse [H, T] and their tolerances, all fp64 on the CPU.

    The tolerances count roundings, with u = 2^-24 the half step of fp32:
      logits   a dot product of d terms of at most S = sum |q_i k_i|: (d + 1) u S scale, and the
               scaled logit (of size at most S scale) is rounded three more times, scale and
               log2(e) as one rounded factor included: (d + 4) u S scale in all
      weights  exp of that, the logit's error as a relative one, and 4 u for exp2 itself; 16-bit
               types round each weight once more, by eps / 2
      sums     n terms, n u of the sum of their magnitudes, in the product and in the normaliser
      output   eps / 2 of its own type
    Weights enter through A = sum w |v| (an output is at most A). f16 weights are kept as
    multiples of 2^-24 after being raised by 2^8, so each is off by at most 2^-33 of the largest
    besides."""
    dt, u = q.dtype, 2.0 ** -24
    half = torch.finfo(dt).eps / 2
    T, H, d = q.shape
    n_kv, n = k.shape[0], k.shape[1]
    q, k, v = q.cpu().double(), k.cpu().double(), v.cpu().double()
    seen = seen.cpu()
    scale = scale if scale > 0 else 1.0 / math.sqrt(d)
    out, lse = torch.zeros(T, H, d, dtype=torch.float64), torch.full((H, T), -math.inf, dtype=torch.float64)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    some = seen.any(1)
    for h in range(H):
        g = h // (H // n_kv)
        z = q[:, h] @ k[g].T * scale
        size = (q[:, h].abs() @ k[g].abs().T * scale).masked_fill(~seen, 0.0).amax(1) if n else torch.zeros(T)
        z = z.masked_fill(~seen, -math.inf)
        m = z.amax(1, keepdim=True) if n else torch.zeros(T, 1)
        m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
        w = torch.exp(z - m)
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
        # a row's sum over the keys that it sees, whatever the others hold
        vg = v[g]
        if torch.isfinite(vg).all():
            out[:, h], big = w @ vg, w @ vg.abs()
        else:
            prod = torch.where(seen[:, :, None], w[:, :, None] * vg[None], torch.zeros(1, dtype=torch.float64))
            out[:, h], big = prod.sum(1), prod.abs().sum(1)
        lse[h] = torch.where(some, m[:, 0] + torch.log(total[:, 0]), lse[h])
        delta = (d + 4) * u * size + 4 * u
        rel = 2 * delta + 2 * n * u + (half if dt != torch.float32 else 2 * u)
        vmax = torch.where(torch.isfinite(vg), vg.abs(), torch.zeros(1, dtype=torch.float64)).amax() if n else 0.0
        out_tol[:, h] = rel[:, None] * big + half * out[:, h].abs() + (n * 2.0 ** -33 * vmax if dt == torch.float16 else 0.0) + 1e-30
        lse_tol[h] = delta + n * u + 4 * u * (torch.where(some, lse[h].abs(), torch.zeros(T, dtype=torch.float64)) + 1)
    return out, lse, out_tol, lse_tol


def check(got, want, tol, what):
    """Equal where the reference is not finite, within tol elsewhere."""
    got = got.cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN at other places"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what + ": infinities"
    over = (got[fine] - want[fine]).abs() / tol[fine]
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 1.0, "%s: %.2f times its tolerance" % (what, worst)
    return worst
