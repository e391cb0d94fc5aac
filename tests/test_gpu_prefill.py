"""ckv_prefill_attention against plain 64-bit attention: packed prompts of every kind of length,
types, layouts, and values that are not finite."""
import itertools
import math

import pytest
import torch

import paper_2508_02401_amd as ckv
from tests.attn_ref import attend, check

pytestmark = pytest.mark.gpu

TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _sums(lens, first=0):
    return list(itertools.accumulate([first] + list(lens)))


def _rand(gen, dt, *shape):
    return torch.randn(shape, generator=gen, dtype=torch.float32).to(dt).cuda()


def _inputs(seed, dt, H, n_kv, d, n, tok_major=True):
    gen = torch.Generator().manual_seed(seed)
    q = _rand(gen, dt, n, H, d)
    if tok_major:
        k, v = (_rand(gen, dt, n, n_kv, d).transpose(0, 1) for _ in range(2))
    else:
        k, v = (_rand(gen, dt, n_kv, n, d) for _ in range(2))
    return q, k, v


def _run(q, k, v, cu, n_kv, scale=0.0, lse=True):
    n, H, d = q.shape
    out = torch.full((n, H, d), 7.0, dtype=q.dtype, device="cuda")
    z = torch.full((H, n), 7.0, dtype=torch.float32, device="cuda") if lse else None
    ckv.ckv_prefill_attention(ckv.attn_desc(H, n_kv, d, q.dtype, scale), q, k, v, cu, out, lse=z)
    torch.cuda.synchronize()
    return out, z


def _check(q, k, v, cu, out, lse, scale=0.0):
    for a, b in zip(cu, cu[1:]):
        if a == b:
            continue
        seen = torch.ones(b - a, b - a, dtype=torch.bool).tril()
        o, z, ot, zt = attend(q[a:b], k[:, a:b], v[:, a:b], seen, scale)
        check(out[a:b], o, ot, "out of %d tokens" % (b - a))
        if lse is not None:
            check(lse[:, a:b], z, zt, "lse of %d tokens" % (b - a))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("H,n_kv,d", [(8, 2, 64), (28, 4, 128), (4, 4, 128), (6, 1, 64)])
def test_lengths(dt, H, n_kv, d):
    # one token, around tiles of 32 and 64 keys and of 256 rows, and more; empty prompts
    lens = [1, 0, 2, 31, 32, 33, 63, 64, 65, 0, 127, 129, 255, 300, 513]
    cu = _sums(lens)
    q, k, v = _inputs(len(lens) * H + d, dt, H, n_kv, d, cu[-1])
    out, lse = _run(q, k, v, cu, n_kv)
    _check(q, k, v, cu, out, lse)


@pytest.mark.parametrize("dt", TYPES)
def test_long(dt):
    cu = _sums([2500])
    q, k, v = _inputs(1, dt, 4, 2, 128, cu[-1])
    out, lse = _run(q, k, v, cu, 2)
    _check(q, k, v, cu, out, lse)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_layouts(dt, d):
    # head-major K and V, rows and heads with gaps, outputs inside a wider buffer
    H, n_kv, cu = 8, 2, _sums([70, 200], first=3)
    n = cu[-1] + 5
    q, k, v = _inputs(2, dt, H, n_kv, d, n, tok_major=False)
    wide = torch.zeros(n, H + 2, d + 16, dtype=dt, device="cuda")
    wide[:, 1:H + 1, :d] = q
    kw = torch.zeros(2, n_kv, n + 3, d + 16, dtype=dt, device="cuda")
    kw[0, :, :n, :d], kw[1, :, :n, :d] = k, v
    ow = torch.full((n, H + 1, d + 32), 5.0, dtype=dt, device="cuda")
    lw = torch.full((H, n + 7), 5.0, dtype=torch.float32, device="cuda")
    ckv.ckv_prefill_attention(ckv.attn_desc(H, n_kv, d, dt, 0.3), wide[:, 1:H + 1, :d],
                              kw[0, :, :n, :d], kw[1, :, :n, :d], cu, ow[:, :H, :d], lse=lw[:, :n])
    torch.cuda.synchronize()
    _check(q, k, v, cu, ow[:, :H, :d], lw[:, :n], 0.3)
    # rows before the first prompt and behind the last one, and the gaps, stay as they were
    assert (ow[:3] == 5.0).all() and (ow[cu[-1]:] == 5.0).all()
    assert (ow[:, H:] == 5.0).all() and (ow[:, :, d:] == 5.0).all()
    assert (lw[:, :3] == 5.0).all() and (lw[:, cu[-1]:] == 5.0).all()


def test_many_prompts():
    # more prompts than one launch takes, many of them empty
    lens = [(7 * i) % 11 for i in range(1000)]
    cu = _sums(lens)
    q, k, v = _inputs(3, torch.bfloat16, 4, 1, 64, cu[-1])
    out, lse = _run(q, k, v, cu, 1)
    _check(q, k, v, cu, out, lse)


def test_no_lse_and_no_tokens():
    q, k, v = _inputs(4, torch.bfloat16, 4, 2, 64, 40)
    with_lse, _ = _run(q, k, v, [0, 40], 2)
    without, _ = _run(q, k, v, [0, 40], 2, lse=False)
    assert torch.equal(with_lse, without)
    untouched, _ = _run(q, k, v, [5, 5, 5], 2)
    assert (untouched == 7.0).all()


@pytest.mark.parametrize("dt", TYPES)
def test_values_that_are_not_finite(dt):
    # a NaN or an infinity reaches the rows from its token on and no earlier one
    cu = _sums([200, 90])
    for at, what in ((0, math.nan), (77, math.inf), (130, -math.inf), (199, math.nan), (210, math.inf)):
        q, k, v = _inputs(5 + at, dt, 4, 2, 64, cu[-1])
        v[1, at, 3] = what
        v[0, at, 5] = -what
        v[0, min(at + 9, 199), 5] = what  # with its opposite: NaN
        out, lse = _run(q, k, v, cu, 2)
        _check(q, k, v, cu, out, lse)
    q, k, v = _inputs(6, dt, 4, 2, 64, cu[-1])
    k[0, 100] = math.nan
    out, lse = _run(q, k, v, cu, 2)
    assert torch.isfinite(out[:100]).all() and torch.isfinite(out[200:]).all()
    assert torch.isnan(out[100:200, :2]).all() and torch.isfinite(out[100:200, 2:]).all()
    assert torch.isnan(lse[:2, 100:200]).all() and torch.isfinite(lse[2:]).all()


@pytest.mark.parametrize("dt", TYPES)
def test_large_logits(dt):
    # maxima that rise along the keys, and one key that outweighs all others
    cu, d = _sums([600]), 128
    q, k, v = _inputs(7, dt, 4, 2, d, cu[-1])
    q = q * 4
    k = k * torch.linspace(0.2, 6, 600, device="cuda").to(dt)[:, None]
    k[:, 350] = q[400].float().mean(0).to(dt) * 3
    out, lse = _run(q, k, v, cu, 2)
    _check(q, k, v, cu, out, lse)


def test_captured_and_replayed():
    cu = _sums([130, 7, 400])
    q, k, v = _inputs(8, torch.float16, 8, 2, 128, cu[-1])
    desc = ckv.attn_desc(8, 2, 128, torch.float16)
    out, lse = torch.zeros_like(q), torch.zeros(8, cu[-1], device="cuda")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ckv.ckv_prefill_attention(desc, q, k, v, cu, out, lse=lse)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ckv.ckv_prefill_attention(desc, q, k, v, cu, out, lse=lse)
    for seed in range(3):
        q2, k2, v2 = _inputs(20 + seed, torch.float16, 8, 2, 128, cu[-1])
        q.copy_(q2), k.copy_(k2), v.copy_(v2)
        out.zero_(), lse.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, want_lse = _run(q, k, v, cu, 2)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)


def test_lse_feeds_the_compression():
    # the window rows' log-sum-exp in place of the scoring's first pass over K: the same scores
    # to the rounding of both, and the very cache where the scores leave no doubt
    H, n_kv, d, w, cu = 8, 2, 128, 32, _sums([700, 333])
    q, k, v = _inputs(9, torch.bfloat16, H, n_kv, d, cu[-1])
    _, lse = _run(q, k, v, cu, n_kv)
    desc = ckv.layer_desc(H, n_kv, d, w)
    mask = [1, 0, 0, 1, 0, 1, 1, 0]
    runs = []
    for use in (False, True):
        seqs = []
        for a, b in zip(cu, cu[1:]):
            s = ckv.Seq(q[b - w:b].transpose(0, 1), k[:, a:b], v[:, a:b], 96,
                        lse=lse[:, b - w:b] if use else None)
            seqs.append(ckv.alloc_outputs(desc, s))
        ckv.ckv_compress_layer(desc, mask, seqs, ckv.alloc_workspace(desc, seqs, "cuda"))
        torch.cuda.synchronize()
        runs.append(seqs)
    for own, given in zip(*runs):
        # the normalisers' logarithms are each off by at most 2.2e-4 (132 roundings of 2^-24 of
        # logits' terms of up to 16 in sum, 700 of the normaliser): a score by twice that and
        # the roundings that both share
        assert ((own.scores - given.scores).abs() <= 5e-4 * own.scores).all()
        for a, b in zip(own.idx, given.idx):
            assert torch.isin(a, b).float().mean() >= 0.9  # neighbours in rank may change places
