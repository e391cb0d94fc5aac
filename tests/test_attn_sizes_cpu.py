"""What bounds of a paged step are refused, and what its workspace grows with (no GPU)."""
import pytest

import paper_2508_02401_amd as ckv
from tests.test_attn_abi_cpu import _attention, _batch, _desc


def _bytes(**kw):
    return ckv.ckv_paged_workspace_bytes(_desc(), _batch(**kw))


@pytest.mark.parametrize("n", [0x7FFFF001, 2 ** 31 - 1])
def test_requests_longer_than_positions_in_32_bits(n):
    assert _attention(batch=_batch(max_kv=n)) == ckv.CKV_ERR_UNSUPPORTED
    assert _bytes(max_kv=n) == 0
    assert _bytes(max_kv=0x7FFFF000) > 0


def test_workspace():
    # nothing to split, split requests of few rows, and of many; a note for every row
    short, long = _bytes(max_kv=100, max_q=1), _bytes(max_kv=5000, max_q=1)
    assert short < 1024 < long < _bytes(max_kv=5000, max_q=100)
    d = _desc()
    assert _bytes(max_kv=5000, max_q=1, total_q=1000) == \
        _bytes(max_kv=5000, max_q=1, total_q=10) + 990 * 8 * d.num_q_heads
