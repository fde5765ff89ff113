"""Ragged attention where single values or single rows decide: a batch with one key in all."""
import numpy as np
import pytest
import torch

from tests.test_gpu_attn_ragged import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head", [(2, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("rows", [1, 3, 40])
@pytest.mark.parametrize("k_lens,slots", [([1], [5]), ([0, 1], [0, 3]), ([0, 0, 1], [2, 0, 1]), ([1, 0], [4, 0])], ids=str)
def test_one_key_in_the_whole_batch(k_lens, slots, rows, heads, kv_heads, head, dtype):
    """The first token of one sequence, in any slot of a cache: its row is found by the slot's start."""
    capacity, slots = 70, np.array(slots)
    q_lens = [rows] * len(k_lens)
    x = make(q_lens, k_lens, heads, kv_heads, head, dtype, buckets=8, seed=20, k_rows=6 * capacity)
    got = check(x, q_lens, k_lens, dtype, causal=True, max_distance=20, k_starts=slots * capacity, training=False)[2]
    b = k_lens.index(1)
    v = x["v"][slots[b] * capacity].repeat_interleave(heads // kv_heads, 0)
    assert torch.equal(got[0][(b + 1) * rows - 1].cpu(), v)  # the last row stands at the key
    x["bias"] = None
    x["key_mask"] = torch.ones(6 * capacity, dtype=torch.uint8)
    x["key_mask"][0] = 0
    check(x, q_lens, k_lens, dtype, k_starts=slots * capacity, training=False)
