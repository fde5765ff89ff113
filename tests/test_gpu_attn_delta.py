"""Query and bias gradients in bfloat16 are good to the rounding of the result where few keys have the weight or a bias adds their errors up.

Bound.  y is what bfloat16 makes of x', which is off the exact x by d.  No other bfloat16 is nearer to x', so |y - x| <= |x rounded - x| + 2 d: in the 2-norm
the exact result's own rounding, which is computed, and 2 |d|.  d: float32's 5e-6 (test_gpu_attn_ragged; times S / 16 where scores are of size S) and 2^-16 of
dS, which are two bfloat16, each of them of the same sums of magnitudes."""
import math

import pytest
import torch

from tests import train_reference as R
from tests.test_gpu_attn_ragged import dev, make

pytestmark = pytest.mark.gpu


def expected(x, lens, causal, bidirectional, bias):
    """(dq, the sum of its terms' sizes), the same of d_bias, size of the scores; all in float64"""
    q, k, v, d, w = (x[n].double() for n in ("q", "k", "v", "d_out", "bias"))
    H, G, D = q.shape[1], k.shape[1], q.shape[2]
    scale = 1 / math.sqrt(D)
    dq, dq_size, dw, dw_size = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(w), torch.zeros_like(w)
    row, most = 0, 0.0
    for n in lens:
        rows = slice(row, row + n)
        far = torch.arange(n)[:, None] - torch.arange(n)[None, :]
        place = torch.tensor([R.bucket(i, w.shape[0], 20, bidirectional) for i in range(-n, n + 1)])[far + n]
        seen = far >= 0 if causal else torch.ones((n, n), dtype=torch.bool)
        if x["key_mask"] is not None:
            seen = seen & (x["key_mask"][rows] != 0)[None, :]
        for h in range(H):
            g = h // (H // G)
            s = q[rows, h] @ k[rows, g].T * scale + (w[place, h] if bias else 0)
            most = max(most, float(s.abs().max()))
            p = torch.nan_to_num(torch.softmax(torch.where(seen, s, torch.full((), -math.inf, dtype=torch.float64)), 1))
            dp = d[rows, h] @ v[rows, g].T
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            dq[rows, h], dq_size[rows, h] = scale * ds @ k[rows, g], scale * ds.abs() @ k[rows, g].abs()
            dw[:, h].index_add_(0, place.reshape(-1), ds.reshape(-1))
            dw_size[:, h].index_add_(0, place.reshape(-1), ds.abs().reshape(-1))
        row += n
    return (dq, dq_size), (dw, dw_size), most


def check(x, lens, causal, bidirectional, bias):
    from paper_2503_05931_amd import training as T
    H, G, D = x["q"].shape[1], x["k"].shape[1], x["q"].shape[2]
    print("case", lens[:6], H, G, D, causal, bidirectional, bias, flush=True)
    plan = T.Attention(lens, lens, H, D, torch.bfloat16, n_kv_heads=G, causal=causal, bias_buckets=8 if bias else 0, bias_max_distance=20, bias_bidirectional=bidirectional)
    d = dev(x)
    extra = dict(bias=d["bias"] if bias else None, key_mask=d["key_mask"])
    out, lse = plan.aed_attn_forward(d["q"], d["k"], d["v"], **extra)
    got = plan.aed_attn_backward(d["d_out"], d["q"], d["k"], d["v"], out, lse, **extra)
    torch.cuda.synchronize()
    dq, dw, most = expected(x, lens, causal, bidirectional, bias)
    for n, g, (want, size) in (("dq", got[0], dq),) + ((("d_bias", got[3], dw),) if bias else ()):
        rounding = float((want.to(torch.bfloat16).double() - want).norm())
        before = (5e-6 * max(1, most / 16) + 2 ** -16) * float(size.norm())
        off = float((g.double().cpu() - want).norm())
        print(f"{n}: off {off / float(want.norm()):.5f}, rounding alone {rounding / float(want.norm()):.5f}, allowed {(rounding + 2 * before) / float(want.norm()):.5f}")
        assert off <= rounding + 2 * before, n


@pytest.mark.parametrize("heads,kv_heads,head", [(2, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("causal,bidirectional", [(True, False), (False, True), (False, False)])
@pytest.mark.parametrize("lens", [[2, 3, 9, 12], [33, 20, 31], [64, 65, 128, 127], [7, 9] * 80, [150, 300]], ids=lambda n: f"{len(n)}x{max(n)}")
@pytest.mark.parametrize("masked", [0.0, 0.3])
def test_with_a_bias(lens, masked, causal, bidirectional, heads, kv_heads, head):
    check(make(lens, lens, heads, kv_heads, head, "bf16", buckets=8, masked=masked, seed=30), lens, causal, bidirectional, True)


@pytest.mark.parametrize("heads,kv_heads,head", [(2, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens", [[2, 3, 9, 12], [33, 20, 31], [64, 65, 128, 127], [7, 9] * 80], ids=lambda n: f"{len(n)}x{max(n)}")
@pytest.mark.parametrize("sharp", [1, 6])
def test_without_one(lens, sharp, causal, heads, kv_heads, head):
    x = make(lens, lens, heads, kv_heads, head, "bf16", buckets=8, seed=31)
    x["q"] *= sharp
    check(x, lens, causal, False, False)
