"""What the paged cache's bindings refuse before anything reaches the library (no GPU)."""
import pytest
import torch

import paper_2508_02401_amd as ckv


def _pool(device="cpu"):
    return torch.zeros(5, 2, 16, 64, dtype=torch.bfloat16, device=device)


def test_pools_on_two_devices():
    for k, v in ((_pool(), _pool("meta")), (_pool("meta"), _pool())):
        with pytest.raises(ValueError, match="device"):
            ckv.paged_cache(k, v)


def test_structs_that_were_filled_by_hand():
    # exported for the C interface; the calls cannot look at the tensors behind their pointers
    desc, pool = ckv.attn_desc(4, 2, 64), _pool()
    cache = ckv.paged_cache(pool, pool)
    ints = torch.zeros(9, dtype=torch.int32)
    batch = ckv.paged_batch(ints[:4], ints[:3], ints.view(3, 3), 9, 4, 9)
    q, k = torch.zeros(9, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 9, 64, dtype=torch.bfloat16)
    bare_cache = ckv.ckv_paged_cache.from_buffer_copy(cache)
    bare_batch = ckv.ckv_paged_batch.from_buffer_copy(batch)
    with pytest.raises(ValueError, match="paged_cache"):
        ckv.ckv_paged_write(desc, bare_cache, k, k, ints)
    with pytest.raises(ValueError, match="paged_cache"):
        ckv.ckv_paged_attention(desc, bare_cache, batch, q, torch.empty_like(q), ints)
    with pytest.raises(ValueError, match="paged_batch"):
        ckv.ckv_paged_attention(desc, cache, bare_batch, q, torch.empty_like(q), ints)


@pytest.mark.parametrize("over", [1 << 32, -(1 << 32), (1 << 32) * 3])
def test_numbers_past_32_bits(over):
    # their low 32 bits alone would be taken for other, valid ones
    desc = ckv.attn_desc(4, 2, 64)
    ints = torch.zeros(9, dtype=torch.int32)
    for bad in ((9 + over, 4, 9), (9, 4 + over, 9), (9, 4, 9 + over)):
        with pytest.raises(ValueError, match="32 bits"):
            ckv.paged_batch(ints[:4], ints[:3], ints.view(3, 3), *bad)
    one = ints[:1]
    with pytest.raises(ValueError, match="32 bits"):
        ckv.ckv_paged_plan(ints[:3], ints[:3], ints.view(3, 3), 16 + over, ints, one, ints[:4], ints[:3], ints, one)
    q, k = torch.zeros(9, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 9, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="cu_seqlens"):
        ckv.ckv_prefill_attention(desc, q, k, k, [0, 4 + over, 9], torch.empty_like(q))


def test_workspaces_with_gaps():
    # its bytes are counted, and written one after the other from its first on
    desc, pool, ints = ckv.attn_desc(4, 2, 64), _pool(), torch.zeros(9, dtype=torch.int32)
    cache, batch = ckv.paged_cache(pool, pool), ckv.paged_batch(ints[:4], ints[:3], ints.view(3, 3), 9, 4, 9)
    q = torch.zeros(9, 4, 64, dtype=torch.bfloat16)
    for ws in (torch.zeros(1).expand(10 ** 6), torch.zeros(2 * 10 ** 5)[::2]):
        with pytest.raises(ValueError, match="contiguous"):
            ckv.ckv_paged_attention(desc, cache, batch, q, torch.empty_like(q), ws)
