"""Ragged attention in the forms that its work lists choose between: whole items and halves, few rows, split keys.  Bounds are those of
test_gpu_attn_ragged (see there)."""
import random

import pytest
import torch

from tests import train_reference as R
from tests.test_gpu_attn_ragged import check, make

pytestmark = pytest.mark.gpu

# sequences x heads: more than 128 items of 128 rows and of 128 keys each, so that none is halved
MANY = dict(heads=8, kv_heads=8, n=18)


def lengths(n, top, keys, seed):
    g = random.Random(seed)
    q, k = [g.randint(0, top) for _ in range(n)], [g.randint(0, keys) for _ in range(n)]
    q[0], k[1], q[2], k[3] = top, keys, 1, 1
    return q, k


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("head", [64, 128])
@pytest.mark.parametrize("top,keys", [(132, 140), (70, 33), (20, 190), (260, 66)])
def test_many_sequences(top, keys, head, dtype):
    q, k = lengths(MANY["n"], top, keys, top)
    check(make(q, k, MANY["heads"], MANY["kv_heads"], head, dtype, masked=0.15 if top == 132 else 0.0, seed=top), q, k, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("head", [64, 128])
@pytest.mark.parametrize("causal,bidirectional,masked", [(True, False, 0.0), (False, True, 0.2), (True, False, 0.2)])
def test_many_sequences_with_bias(causal, bidirectional, masked, head, dtype):
    q, _ = lengths(MANY["n"], 150, 1, 7)
    check(make(q, q, 8, 8, head, dtype, buckets=16, masked=masked, seed=8), q, q, dtype, causal=causal, max_distance=64, bidirectional=bidirectional)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("head", [64, 128])
def test_many_sequences_causal_with_shared_heads(head, dtype):
    q, _ = lengths(24, 140, 1, 9)
    k = [n + (i % 3) * 20 for i, n in enumerate(q)]  # rows stand at the last keys
    check(make(q, k, 16, 8, head, dtype, seed=10), q, k, dtype, causal=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("head", [64, 128])
@pytest.mark.parametrize("q,k", [([40, 3, 64], [1500, 1100, 1024]), ([130, 5], [1300, 2100]), ([1, 16], [2048, 1030]), ([17, 32], [900, 1090])], ids=str)
def test_split_keys(q, k, head, dtype):
    x = make(q, k, 2, 1, head, dtype, masked=0.2, seed=11)
    x["key_mask"][300:900] = 0  # a part without a visible key
    check(x, q, k, dtype, training=False)
    check(make(q, k, 2, 2, head, dtype, buckets=32, seed=12), q, k, dtype, causal=True, max_distance=128, training=False)


@pytest.mark.parametrize("rows", [1, 16, 17, 33, 65])
@pytest.mark.parametrize("slope", [0.03, 0.5, -0.5])
def test_scores_that_grow_or_fall_along_the_keys(slope, rows):
    """Every step of the walk has a new maximum, or none but the first; the last keys outweigh all others, or the first.  A score of size S is
    the sum of 64 products, one of which is nearly all of it: 64 roundings of S at the most, one more in units of log2 e and one in its distance to the
    maximum.  Weights are off by a factor of up to exp(e), e = 66 S 2^-24, and by as much again in their sum."""
    from paper_2503_05931_amd import training as T
    q, k = [rows, rows], [400, 1200]
    x = make(q, k, 2, 2, 64, "fp32", seed=13)
    place = torch.cat([torch.arange(n, dtype=torch.float32) for n in k])
    x["q"][..., 0] = 8.0
    x["k"][..., 0] = slope * place[:, None]  # scores move by slope a key
    plan = T.Attention(q, k, 2, 64, torch.float32, scale=0.125)
    out, lse = (t.cpu().double() for t in plan.aed_attn_forward(x["q"].cuda(), x["k"].cuda(), x["v"].cuda()))
    wide = [x[n].double() for n in ("q", "k", "v")]
    want, want_lse = R.attention(*wide, q, k, scale=0.125)
    size, _ = R.attention(wide[0], wide[1], wide[2].abs(), q, k, scale=0.125)  # sum of p |v|
    most = 0.125 * max((wide[0][a:a + n, h] @ wide[1][b:b + m, h].T).abs().max() for h in range(2)
                       for a, n, b, m in ((0, q[0], 0, k[0]), (q[0], q[1], k[0], k[1])))
    e = float(66 * most * 2 ** -24)
    assert float(((out - want).abs() - 2 * e * size).max()) <= 5e-6 * float(want.abs().max())
    assert float((lse - want_lse).abs().max()) <= 2 * e


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("head", [64, 128])
@pytest.mark.parametrize("form", ["whole", "halves", "few", "split", "bias"])
def test_what_masked_places_hold_does_not_matter(form, head, dtype):
    """The same bits, whatever masked keys and values are: NaN, infinities, the type's largest."""
    from paper_2503_05931_amd import training as T
    n, top, keys, heads = dict(whole=(18, 132, 150, 8), halves=(5, 100, 70, 2), few=(20, 3, 200, 8), split=(4, 70, 1500, 2), bias=(18, 132, 0, 8))[form]
    q, k = lengths(n, top, max(keys, 1), 3)
    k = k if keys else q
    training = form != "split"
    plan = T.Attention(q, k, heads, head, dtype, causal=form == "bias", bias_buckets=16 if form == "bias" else 0, bias_max_distance=64, training=training)
    g = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
    x, kk, vv, d, bias = rnd(sum(q), heads, head), rnd(sum(k), heads, head), rnd(sum(k), heads, head), rnd(sum(q), heads, head), rnd(16, heads)
    mask = (torch.rand(sum(k), generator=g, device="cuda") > 0.3).to(torch.uint8)
    if form == "split":
        mask[100:700] = 0
    seen = []
    for bad in (0.0, float("nan"), float("inf"), -float("inf"), torch.finfo(dtype).max):
        a, b = kk.clone(), vv.clone()
        a[mask == 0] = bad
        b[mask == 0] = bad
        extra = dict(bias=bias if form == "bias" else None, key_mask=mask)
        out, lse = plan.aed_attn_forward(x, a, b, **extra)
        got = [out, lse]
        if training:
            got += [t for t in plan.aed_attn_backward(d, x, a, b, out, lse, **extra) if t is not None]
        seen.append([t.clone() for t in got])
        assert all(torch.isfinite(t.float()).all() for i, t in enumerate(seen[-1]) if i != 1)
        assert all(torch.equal(s, t) for s, t in zip(seen[0], seen[-1]))
        if training:
            assert (seen[-1][3][mask == 0] == 0).all() and (seen[-1][4][mask == 0] == 0).all()
    torch.cuda.synchronize()
