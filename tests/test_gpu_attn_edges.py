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


def apart(t, row, head):
    """A copy of [rows, heads, D] with these strides; what lies between holds anything."""
    rows, heads, _ = t.shape
    place = torch.empty((rows - 1) * row + (heads - 1) * head + t.shape[2], dtype=t.dtype, device="cuda")
    far = place.as_strided(t.shape, (row, head, 1))
    far.copy_(t)
    return far


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("head_stride", [(1 << 27) + 8, (1 << 30) + 64])
def test_heads_far_apart(head_stride, dtype):
    """Heads outermost, as in a tensor of a million rows or more: byte offsets past 32 bits."""
    lens = [33, 40]
    x = make(lens, lens, 2, 2, 64, dtype, seed=26)
    d = {n: None if t is None else apart(t.cuda(), 64, head_stride) if t.dim() == 3 else t.cuda() for n, t in x.items()}
    check(x, lens, lens, dtype, causal=True, on=d)


@pytest.mark.parametrize("rows", [1, 40])
def test_a_cache_past_32_bits(rows):
    """Slots 2^25 rows into a cache: 4.3 GB from its beginning."""
    slot, k_lens = 1 << 25, [200, 1]
    starts = np.array([slot, slot + 300])
    x = make([rows] * 2, k_lens, 2, 2, 64, "bf16", seed=27, k_rows=501)
    d = {n: None if t is None else t.cuda() for n, t in x.items()}
    for n in ("k", "v"):
        wide = torch.empty((slot + 501, 2, 64), dtype=torch.bfloat16, device="cuda")
        wide[slot:] = d[n]
        d[n] = wide
    from paper_2503_05931_amd import training as T
    plan = T.Attention([rows] * 2, k_lens, 2, 64, torch.bfloat16, k_starts=starts, training=False)
    check(x, [rows] * 2, k_lens, "bf16", k_starts=starts - slot, training=False, plan=plan, on=d)


def test_outputs_whose_vectors_share_elements_are_refused():
    import ctypes as C
    from paper_2503_05931_amd import binding, training as T
    x = make([3, 4], [3, 4], 2, 2, 64, "bf16", seed=28)
    d = {n: t.cuda() for n, t in x.items() if t is not None}
    plan = T.Attention([3, 4], [3, 4], 2, 64, torch.bfloat16, training=False)
    out, lse = plan.aed_attn_forward(d["q"], d["k"], d["v"])
    wide = torch.zeros(7 * 512, dtype=torch.bfloat16, device="cuda")
    rows = [T.AedRows(d[n].data_ptr(), 128, 64) for n in ("q", "k", "v")]
    for row, head, status in ((64, 64, binding.AED_EINVAL), (128, 128, binding.AED_EINVAL), (128, 96, binding.AED_EINVAL), (64, 448, 0), (128, 64, 0), (512, 72, 0)):
        to = T.AedRows(wide.data_ptr(), row, head)
        assert plan.lib.aed_attn_forward(plan.handle, *rows, None, None, to, C.c_void_p(lse.data_ptr())) == status, (row, head)
        torch.cuda.synchronize()
        if status == 0:
            assert torch.equal(wide.as_strided((7, 2, 64), (row, head, 1)), out)
