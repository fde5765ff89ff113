"""Key and value gradients in bfloat16 are good to the rounding of the result in small batches of few rows, where the roundings of a handful of weights do not
average out.  Bound: that of test_gpu_attn_delta, with 2^-16 of the weights and of dS, which are two bfloat16 each."""
import math

import pytest
import torch

from tests.test_gpu_attn_ragged import dev, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads,head", [(2, 2, 64), (8, 2, 128), (8, 1, 128)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("q_lens,k_lens", [([4], [119]), ([10], [10]), ([3, 0, 6, 5], [77, 4, 130, 90]), ([64, 1], [64, 300]), ([1], [3])], ids=str)
def test_few_rows(q_lens, k_lens, causal, heads, kv_heads, head):
    from paper_2503_05931_amd import training as T
    x = make(q_lens, k_lens, heads, kv_heads, head, "bf16", seed=32)
    print("case", q_lens, k_lens, heads, kv_heads, head, causal, flush=True)
    plan = T.Attention(q_lens, k_lens, heads, head, torch.bfloat16, n_kv_heads=kv_heads, causal=causal)
    d = dev(x)
    out, lse = plan.aed_attn_forward(d["q"], d["k"], d["v"])
    _, dk, dv, _ = plan.aed_attn_backward(d["d_out"], d["q"], d["k"], d["v"], out, lse)
    torch.cuda.synchronize()
    q, k, v, g_out = (x[n].double() for n in ("q", "k", "v", "d_out"))
    scale, most = 1 / math.sqrt(head), 0.0
    want, size = ([torch.zeros_like(k), torch.zeros_like(k)] for _ in range(2))
    row = at = 0
    for nq, nk in zip(q_lens, k_lens):
        qs, ks = slice(row, row + nq), slice(at, at + nk)
        seen = torch.arange(nq)[:, None] + nk - nq >= torch.arange(nk)[None, :] if causal else torch.ones((nq, nk), dtype=torch.bool)
        for h in range(heads if nq else 0):
            g = h // (heads // kv_heads)
            s = q[qs, h] @ k[ks, g].T * scale
            most = max(most, float(s.abs().max()))
            p = torch.nan_to_num(torch.softmax(torch.where(seen, s, torch.full((), -math.inf, dtype=torch.float64)), 1))
            dp = g_out[qs, h] @ v[ks, g].T
            ds = scale * p * (dp - (p * dp).sum(1, keepdim=True))
            want[0][ks, g] += ds.T @ q[qs, h]
            size[0][ks, g] += ds.abs().T @ q[qs, h].abs()
            want[1][ks, g] += p.T @ g_out[qs, h]
            size[1][ks, g] += p.T @ g_out[qs, h].abs()
        row += nq
        at += nk
    for n, got, w, m in zip(("dk", "dv"), (dk, dv), want, size):
        rounding = float((w.to(torch.bfloat16).double() - w).norm())
        before = (5e-6 * max(1, most / 16) + 2 ** -16) * float(m.norm())
        off = float((got.double().cpu() - w).norm())
        print(f"{n}: off {off / float(w.norm()):.5f}, rounding alone {rounding / float(w.norm()):.5f}, allowed {(rounding + 2 * before) / float(w.norm()):.5f}")
        assert off <= rounding + 2 * before, n
