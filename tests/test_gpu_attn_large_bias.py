"""Bias tables whose entries are large: weights stay weights, forward and backward, whatever the size of a row's scores.

Bounds.  u = 2^-24.  A score is a product of head_dim terms and one rounding at its own size S, its exponent two more; the weights' sum is one of n
terms, its logarithm, of size log2 n, is good to an ulp, and so are the weight's power of two and its product: a weight is off by
e = 2 u (head_dim P + 6 S + log2 n + 3) + n u of itself, P the largest sum of |q_c k_c| times the scale.  Rows whose scores are beyond a thousand have queries of zeros
here: their scores are table entries, exactly, and S does not enter.  What is made of the weights is off by as much of the same formulas with magnitudes in
the place of numbers, and by u for each of the terms that are added up.  bfloat16: 2^-8 more for the weights, the output in delta, and the result.
"""
import math

import pytest
import torch

from tests import train_reference as R
from tests.test_gpu_attn_ragged import TYPE, dev, make

pytestmark = pytest.mark.gpu

LIMIT = torch.finfo(torch.float32).max / math.log2(math.e)  # finite entries count as no more than that


def expected(x, q_lens, k_lens, dtype, causal, max_distance, bidirectional):
    """name -> (value in float64, how far it may be off)"""
    q, k, v, d = (x[n].double() for n in ("q", "k", "v", "d_out"))
    w = x["bias"].double()
    w = torch.where(torch.isfinite(w), w.clamp(-LIMIT, LIMIT), w)
    H, G, D = q.shape[1], k.shape[1], q.shape[2]
    scale, u, round16 = 1 / math.sqrt(D), 2.0 ** -24, 2.0 ** -8 if dtype == "bf16" else 0.0
    names = dict(out=q, lse=q[..., 0], dq=q, dk=k, dv=v, d_bias=w)
    value, near = ({n: torch.zeros_like(t) for n, t in names.items()} for _ in range(2))
    row = at = 0
    for nq, nk in zip(q_lens, k_lens):
        qs, ks = slice(row, row + nq), slice(at, at + nk)
        far = torch.arange(nq)[:, None] + nk - nq - torch.arange(nk)[None, :]
        place = torch.tensor([R.bucket(n, w.shape[0], max_distance, bidirectional) for n in range(-max(nq, nk), max(nq, nk) + 1)])[far + max(nq, nk)]
        seen = far >= 0 if causal else torch.ones((nq, nk), dtype=torch.bool)
        if x["key_mask"] is not None:
            seen = seen & (x["key_mask"][ks] != 0)[None, :]
        for h in range(H):
            g = h // (H // G)
            s = torch.where(seen, q[qs, h] @ k[ks, g].T * scale + w[place, h], torch.full((), -math.inf, dtype=torch.float64))
            top = s.max(1, keepdim=True).values if nk else torch.full((nq, 1), -math.inf, dtype=torch.float64)
            size = torch.where(top.abs() < 1e3, top.abs() + 30, torch.zeros(()))  # (what is 30 below the top has no weight)
            e = 2 * u * (D * scale * (q[qs, h].abs() @ k[ks, g].abs().T).amax(1, keepdim=True) + 6 * size + math.log2(nk) + 3) + nk * u if nk else top
            p = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
            total = p.sum(1, keepdim=True)
            p = p / torch.where(total == 0, 1.0, total)
            out, do, vv, va = p @ v[ks, g], d[qs, h], v[ks, g], v[ks, g].abs()
            value["out"][qs, h], near["out"][qs, h] = out, (2 * e + nk * u + round16) * (p @ va) + round16 * out.abs()
            value["lse"][qs, h] = (top + torch.log(total))[:, 0]
            near["lse"][qs, h] = (e + 4 * u * (1 + top.abs()))[:, 0]
            ds = p * (do @ vv.T - (do * out).sum(1, keepdim=True))
            a = do.abs() @ va.T
            c = 3 * e + (2 * nk + nq + 2 * D) * u + 2 * round16
            m = c * p * (a + 3 * (p * a).sum(1, keepdim=True))
            value["dq"][qs, h], near["dq"][qs, h] = scale * ds @ k[ks, g], scale * m @ k[ks, g].abs()
            value["dk"][ks, g] += scale * ds.T @ q[qs, h]
            near["dk"][ks, g] += scale * m.T @ q[qs, h].abs()
            value["dv"][ks, g] += p.T @ do
            near["dv"][ks, g] += ((2 * e + nq * u + round16) * p).T @ do.abs()
            value["d_bias"][:, h].index_add_(0, place[seen], ds[seen])
            near["d_bias"][:, h].index_add_(0, place[seen], m[seen])
        row += nq
        at += nk
    for n in ("dq", "dk", "dv", "d_bias"):
        near[n] += round16 * value[n].abs()
    return {n: (value[n], near[n]) for n in names}


def check(x, q_lens, k_lens, dtype, causal=False, max_distance=20, bidirectional=False):
    from paper_2503_05931_amd import training as T
    H, G, D = x["q"].shape[1], x["k"].shape[1], x["q"].shape[2]
    print("case", q_lens[:6], k_lens[:6], H, G, D, dtype, causal, bidirectional, flush=True)
    plan = T.Attention(q_lens, k_lens, H, D, TYPE[dtype], n_kv_heads=G, causal=causal, bias_buckets=x["bias"].shape[0], bias_max_distance=max_distance,
                       bias_bidirectional=bidirectional)
    d = dev(x)
    out, lse = plan.aed_attn_forward(d["q"], d["k"], d["v"], bias=d["bias"], key_mask=d["key_mask"])
    got = (out, lse) + plan.aed_attn_backward(d["d_out"], d["q"], d["k"], d["v"], out, lse, bias=d["bias"], key_mask=d["key_mask"])
    torch.cuda.synchronize()
    worst = {}
    for (n, (want, near)), g in zip(expected(x, q_lens, k_lens, dtype, causal, max_distance, bidirectional).items(), got):
        g = g.double().cpu()
        same = (g == want) | ((g - want).abs() <= near)
        assert bool(same.all()), (n, int((~same).sum()), g.numel(), g[~same][:4], want[~same][:4])
        fine = torch.isfinite(want)
        worst[n] = float(((g - want).abs()[fine] / near[fine].clamp(min=1e-300)).max()) if bool(fine.any()) else 0.0
    print({n: "%.2f" % r for n, r in worst.items()})


LENGTHS = [[1, 3, 33], [70, 9], [150, 2, 100]]
FORMS = [(True, False), (False, True), (False, False)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head", [(2, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("causal,bidirectional", FORMS)
@pytest.mark.parametrize("lens", LENGTHS, ids=str)
def test_a_constant_of_a_hundred(lens, causal, bidirectional, heads, kv_heads, head, dtype):
    """A constant in the table changes no weight, and e^100 is past float32: rows that a tile lacks may not add what they do not have."""
    x = make(lens, lens, heads, kv_heads, head, dtype, buckets=8, seed=21)
    x["bias"] = (x["bias"] + 100).to(TYPE[dtype])
    check(x, lens, lens, dtype, causal, 20, bidirectional)


def whole(x, value):
    """The same entry for all distances; queries of zeros: a row's scores are equal."""
    x["bias"][:] = value
    x["q"][:] = 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head", [(2, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("causal,bidirectional", FORMS)
@pytest.mark.parametrize("value", ["lowest", "largest", -1e9, -1e6, 3e4])
def test_rows_that_see_a_large_bias_only(value, causal, bidirectional, heads, kv_heads, head, dtype):
    """Every key of a row has the same large bias: equal weights that add up to one, and their gradients."""
    q_lens, k_lens = [70, 1, 150], [70, 40, 130]
    value = {"lowest": torch.finfo(TYPE[dtype]).min, "largest": torch.finfo(TYPE[dtype]).max}.get(value, value)
    x = make(q_lens, k_lens, heads, kv_heads, head, dtype, buckets=8, masked=0.2, seed=22)
    whole(x, value)
    check(x, q_lens, k_lens, dtype, causal, 20, bidirectional)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("heads,kv_heads,head", [(2, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("causal,bidirectional", FORMS)
@pytest.mark.parametrize("value", ["lowest", -1e9])
@pytest.mark.parametrize("many", [False, True])
def test_a_bucket_as_good_as_masked(many, value, causal, bidirectional, heads, kv_heads, head, dtype):
    """The bucket of the query's own place has a value that no other key's weight survives beside, and rows that see no other key: the first of a causal
    sequence, the first of a sequence whose keys behind the query share that bucket, and rows whose other keys are masked."""
    lens = [90, 1, 2, 64, 133] + [131, 140, 5, 64] * (9 if many else 0)  # many: whole items, not halves
    x = make(lens, lens, heads, kv_heads, head, dtype, buckets=8, seed=23)
    x["bias"][0] = torch.finfo(TYPE[dtype]).min if value == "lowest" else value
    if bidirectional:
        x["bias"][4] = x["bias"][0]
    x["key_mask"] = torch.ones(sum(lens), dtype=torch.uint8)
    x["key_mask"][20:70] = 0
    x["key_mask"][:12] = 0  # causal: rows up to the 20th see keys 12 on, rows 12 itself only
    at = 0
    for n in lens:  # rows that see keys of that bucket only have scores that are equal
        far = torch.arange(n)[:, None] - torch.arange(n)[None, :]
        seen = (far >= 0 if causal else torch.ones((n, n), dtype=torch.bool)) & (x["key_mask"][at:at + n] != 0)[None, :]
        other = seen & ((far != 0) if bidirectional or causal else far > 0)
        x["q"][at:at + n][~other.any(1)] = 0
        at += n
    check(x, lens, lens, dtype, causal, 20, bidirectional)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("head", [64, 128])
@pytest.mark.parametrize("q_lens,k_lens", [([1, 1, 1], [5, 300, 64]), ([3, 16], [40, 200]), ([40, 100], [1500, 1100]), ([1], [5000])], ids=str)
def test_equal_scores_in_the_other_forms(q_lens, k_lens, head, dtype):
    """Few rows, split keys: the mean of the values, and its lse."""
    from paper_2503_05931_amd import training as T
    x = make(q_lens, k_lens, 2, 2, head, dtype, buckets=8, masked=0.2, seed=24)
    whole(x, torch.finfo(TYPE[dtype]).min)
    plan = T.Attention(q_lens, k_lens, 2, head, TYPE[dtype], bias_buckets=8, bias_max_distance=20, training=False)
    d = dev(x)
    got = plan.aed_attn_forward(d["q"], d["k"], d["v"], bias=d["bias"], key_mask=d["key_mask"])
    want = expected(x, q_lens, k_lens, dtype, False, 20, False)
    for n, g in zip(("out", "lse"), got):
        g = g.double().cpu()
        same = (g == want[n][0]) | ((g - want[n][0]).abs() <= want[n][1])
        assert bool(same.all()), (n, g[~same][:4], want[n][0][~same][:4])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_minus_infinity_is_not_seen(dtype):
    """An entry of minus infinity takes its pairs out: rows that see no others are rows that see nothing."""
    lens = [50, 33]
    x = make(lens, lens, 2, 2, 64, dtype, buckets=8, seed=25)
    x["bias"][0] = -math.inf
    check(x, lens, lens, dtype, True)
