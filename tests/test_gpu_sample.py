"""Sampling (aed_sample) against its definition in float64.

Tokens have to be equal: the weights are float64 exponentials rounded at 2^-44 or finer, so a border lies within 1e-12 of the reference's, and no
number drawn here comes that near to one (exact ties, which powers of two make, are exact on both sides).  logp is a float32 of a float64: half a
step, 2^-24 of it, and 1e-9 for the weights' rounding.
"""
import math

import numpy as np
import pytest
import torch

from paper_2503_05931_amd import binding
from tests import vocab_reference as R

pytestmark = pytest.mark.gpu

TYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}
FILTERS = [dict(), dict(t=0.7), dict(t=0.0), dict(top_k=1), dict(top_k=5, t=1.3), dict(top_k=50, top_p=0.9, t=0.8), dict(top_p=0.5), dict(top_p=0.95, t=2.0),
           dict(min_p=0.1), dict(min_p=0.02, top_p=0.8), dict(top_k=300), dict(top_k=700, top_p=0.99, min_p=0.001, t=1.5), dict(top_p=0.0), dict(min_p=1.0)]


def draw(z, u, dtype, **how):
    from paper_2503_05931_amd import vocabulary as L
    tokens, logp = L.Sampler(z.shape[1], TYPE[dtype]).aed_sample(z.cuda(), u.cuda(), **{"temperature" if n == "t" else n: v for n, v in how.items()})
    torch.cuda.synchronize()
    return tokens.cpu(), logp.cpu()


def check(z, u, dtype, **how):
    print("case", tuple(z.shape), dtype, how, flush=True)
    z = z.to(TYPE[dtype])
    tokens, logp = draw(z, u, dtype, **how)
    zs = z.float().numpy()
    exact = {n: float(np.float32(v)) if n != "top_k" else v for n, v in how.items()}
    for r in range(z.shape[0]):
        token, lp = R.sample(zs[r], float(u[r]), **exact)
        assert int(tokens[r]) == token, (r, int(tokens[r]), token, zs[r][token], float(u[r]))
        assert float(logp[r]) == lp or abs(float(logp[r]) - lp) <= 2 ** -24 * abs(lp) + 1e-9, (r, float(logp[r]), lp)
    return tokens, logp


def rows(n, vocab, seed=0, likely=True):
    g = torch.Generator().manual_seed(seed)
    z = 2 * torch.randn((n, vocab), generator=g)
    if likely:
        z.scatter_add_(1, torch.randint(0, vocab, (n, 6), generator=g), 10 * torch.rand((n, 6), generator=g))
    return z, torch.rand(n, generator=g)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 63, 64, 255, 256, 257, 300, 511, 513, 1000, 4096, 4097, 9001])
def test_vocabularies(vocab, dtype):
    for i, how in enumerate(FILTERS):
        check(*rows(3, vocab, seed=100 * i + vocab), dtype, **how)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [32768, 33001, 65541, 131073, 262144])
def test_wide_vocabularies(vocab, dtype):
    for i, how in enumerate((dict(), dict(top_k=50, top_p=0.9), dict(top_p=0.9), dict(top_k=1000, top_p=0.9, t=1.5))):
        check(*rows(1, vocab, seed=vocab + i), dtype, **how)


@pytest.mark.parametrize("how", FILTERS, ids=str)
def test_flat_rows(how):
    """A model that knows nothing: the nucleus is most of the vocabulary, and borders lie close."""
    z, u = rows(8, 4096, seed=7, likely=False)
    check(0.05 * z, u, "fp32", **how)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [200, 2048, 5000])
def test_equal_logits(vocab, dtype):
    """Rows of one value and of two: filters end inside of equal ones, and take the lowest ids."""
    u = torch.tensor([0.0, 0.25, 0.5, 0.999])
    for z in (torch.full((4, vocab), 1.5), (torch.arange(vocab) % 2).float().repeat(4, 1), -(torch.arange(vocab) % 3).float().repeat(4, 1)):
        for how in (dict(), dict(top_k=3), dict(top_k=120), dict(top_k=130), dict(top_p=0.5), dict(top_p=0.25, top_k=150), dict(min_p=0.5), dict(top_p=2 ** -20), dict(t=0.0)):
            check(z, u, dtype, **how)


def lacking(vocab, dtype):
    z, u = rows(12, vocab, seed=3)
    z = z.to(TYPE[dtype])
    g = torch.Generator().manual_seed(4)
    out = torch.rand(z.shape, generator=g) < 0.9
    out[:, 5] = False
    z[0:2][out[0:2]] = -math.inf
    z[2:4][out[2:4]] = math.nan
    z[4:6][out[4:6]] = torch.finfo(TYPE[dtype]).min
    z[6] = -math.inf
    z[7] = math.nan
    z[8] = -math.inf
    z[8, vocab - 1] = -3.0
    z[9] = torch.finfo(TYPE[dtype]).min
    z[10, 17] = math.inf
    z[11, 17:40] = math.inf
    return z, u


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_that_lack_logits(dtype):
    """Minus infinity, NaN and the type's lowest value in masked places; infinite logits; rows that have nothing left."""
    z, u = lacking(700, dtype)
    for how in FILTERS:
        check(z, u, dtype, **how)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [6000, 20000, 40003])
def test_wide_rows_that_lack_logits(vocab, dtype):
    z, u = lacking(vocab, dtype)
    for how in (dict(), dict(top_k=5), dict(top_p=0.9), dict(min_p=0.01), dict(top_k=700, top_p=0.99, min_p=0.001, t=1.5), dict(top_p=0.8, min_p=0.02)):
        check(z, u, dtype, **how)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [255, 4096])
def test_many_rows(vocab, dtype):
    """More rows than have many wavefronts each: every filter, and the same bits as with a few rows at a time."""
    z, u = rows(601, vocab, seed=5)
    z = z.to(TYPE[dtype])
    z[:12] = lacking(vocab, dtype)[0]
    z[12:16], z[16] = 0.05 * z[12:16], 1.5
    z[17] = (torch.arange(vocab) % 3).to(z.dtype)
    z[18, vocab // 2:] = -math.inf
    for how in FILTERS:
        tokens, logp = draw(z, u, dtype, **how)
        few = check(z[:24], u[:24], dtype, **how)
        parts = few, draw(z[24:300], u[24:300], dtype, **how), draw(z[300:], u[300:], dtype, **how)
        assert all(torch.equal(whole, torch.cat(part)) for whole, part in zip((tokens, logp), zip(*parts)))


def test_uniforms():
    """A row's tokens in turn, and numbers at and beyond the ends."""
    z, _ = rows(1, 300, seed=9)
    for how in (dict(), dict(top_k=20), dict(top_p=0.9)):
        check(z.repeat(400, 1), torch.linspace(0, 1 - 2 ** -24, 400), "fp32", **how)
    z[0, 0] = z[0, 299] = 3.0
    check(z.repeat(6, 1), torch.tensor([0.0, 1 - 2 ** -24, 1.0, 7.0, -1.0, math.nan]), "fp32")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,far", [(300, (5, 15, 25, 33)), (4096, (5, 15, 25, 33)), (9001, (25, 30)), (65541, (15, 28)), (262144, (15, 28))])
def test_unlikely_tokens(vocab, far, dtype):
    """A number of 0 draws the first id, whose weight may be a few multiples of what weights are rounded to: its logp comes from its logit.  Of what is left the
    sum is rounded by 2^-45 a logit at most, 1e-11 of it here and less, as roundings have either sign.  An id that weighs less than half of a multiple is not
    drawn: at t = 0.9, 33 from the largest, 2^-52.9 of multiples of 2^-50, and from 28 on 2^-44.9 of such of 2^-44 and 2^-45.  Then the next one is."""
    bits = 50 if vocab <= 4096 else 62 - (vocab - 1).bit_length()
    for d in far:
        z, _ = rows(3, vocab, seed=vocab + d)
        z[:, 0] = z[:, 1:].max(1).values + 1 - d - torch.tensor([0.0, 0.3, 0.7])
        z[:, 1:] += 1
        for how in (dict(), dict(t=0.9, min_p=1e-30), dict(top_k=vocab - 1), dict(top_p=1 - 2 ** -24)):
            below = z.to(TYPE[dtype]).double()
            below = (below[:, 0] - below.max(1).values) / how.get("t", 1.0) / math.log(2) < -bits - 1
            tokens, logp = check(torch.where(below[:, None] & (torch.arange(vocab) == 0), -math.inf, z), torch.zeros(3), dtype, **how)
            again = draw(z.to(TYPE[dtype]), torch.zeros(3), dtype, **how)
            assert torch.equal(tokens, again[0]) and torch.equal(logp, again[1])
        z[:, 20:] = -math.inf
        for how in (dict(top_k=20), dict(top_k=40, top_p=1 - 2 ** -24), dict(top_p=1 - 2 ** -24)):
            check(z, torch.zeros(3), dtype, **how)


def test_extreme_temperatures_and_logits():
    z, u = rows(6, 1000, seed=11)
    for t in (1e-38, 1e-3, 100.0, 3e38):
        check(z, u, "fp32", t=t)
        check(z, u, "fp32", t=t, top_p=0.9)
    check(z * 1e37, u, "fp32", t=1.0)
    check(z * 1e37, u, "fp32", t=1e37, top_p=0.7)
    check(z * 1e-30, u, "fp32", t=1e-30, top_p=0.7)
    check(z + 1e6, u, "fp32", top_k=600)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_parameters_by_row(dtype):
    """Every row with its own, ones that are out of their range among them."""
    from paper_2503_05931_amd import vocabulary as L
    z, u = rows(40, 1500, seed=13)
    z = z.to(TYPE[dtype])
    pick = lambda *v: [v[i % len(v)] for i in range(40)]  # noqa: E731
    t, k = pick(1.0, 0.0, 0.5, -2.0, math.nan, 1.7, math.inf), pick(0, 3, -4, 50, 1500, 2000, 1, 900)
    p, m = pick(1.0, 0.9, 0.3, 5.0, math.nan, -1.0, 0.0, 0.8, 0.99), pick(0.0, 0.0, -3.0, 0.05, 0.0, math.nan, 0.0, 0.001, 0.0, 7.0, 0.0)
    f32 = lambda v: torch.tensor(v, dtype=torch.float32)  # noqa: E731
    plan = L.Sampler(1500, TYPE[dtype])
    tokens, logp = plan.aed_sample(z.cuda(), u.cuda(), temperature=f32(t).cuda(), top_k=torch.tensor(k, dtype=torch.int32).cuda(), top_p=f32(p).cuda(), min_p=f32(m).cuda())
    for r in range(40):
        tt = t[r] if t[r] > 0 else 0.0
        how = dict(t=np.float32(tt), top_k=max(k[r], 0), top_p=np.float32(p[r]) if p[r] < 1 else 1.0, min_p=np.float32(m[r]) if m[r] > 0 else 0.0)
        token, lp = R.sample(z[r].float().numpy(), float(u[r]), **how)
        assert int(tokens[r]) == token, (r, how)
        assert abs(float(logp[r]) - lp) <= 2 ** -24 * abs(lp) + 1e-9, (r, how)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pitch,skip", [(1024, 0), (1003, 1), (1005, 2), (2000, 3)])
def test_row_strides(pitch, skip, dtype):
    from paper_2503_05931_amd import vocabulary as L
    z, u = rows(9, 1001, seed=pitch)
    wide = torch.full((9, pitch + 8), 100.0, dtype=TYPE[dtype])  # what lies beside a row would be drawn
    flat = wide.flatten()[:9 * pitch + skip]
    view = flat.as_strided((9, 1001), (pitch, 1), skip)
    flat.fill_(100.0)
    view.copy_(z)
    z = view.clone()
    device = flat.cuda()
    plan = L.Sampler(1001, TYPE[dtype])
    for how in (dict(temperature=1.0), dict(top_k=40), dict(top_p=0.9), dict(top_p=0.999, temperature=3.0)):
        a = plan.aed_sample(z.cuda(), u.cuda(), **how)
        b = plan.aed_sample(device.as_strided((9, 1001), (pitch, 1), skip), u.cuda(), **how)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(device.cpu(), flat)


def test_offsets_past_32_bits():
    from paper_2503_05931_amd import vocabulary as L
    z, u = rows(3, 900, seed=21)
    far = torch.empty(3 * (1 << 30), dtype=torch.bfloat16, device="cuda").as_strided((3, 900), (1 << 30, 1))
    far.copy_(z)
    plan = L.Sampler(900, torch.bfloat16)
    a, b = plan.aed_sample(far, u.cuda(), top_p=0.9), plan.aed_sample(far.contiguous(), u.cuda(), top_p=0.9)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_same_bits_in_a_graph_and_on_another_stream():
    from paper_2503_05931_amd import vocabulary as L
    z, u = rows(64, 4096, seed=31)
    z, u = z.cuda(), u.cuda()
    how = dict(temperature=torch.rand(64, device="cuda") * 2, top_p=torch.rand(64, device="cuda"), top_k=torch.randint(0, 600, (64,), dtype=torch.int32, device="cuda"))
    first = L.Sampler(4096, torch.float32).aed_sample(z, u, **how)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        plan = L.Sampler(4096, torch.float32)
    again = plan.aed_sample(z, u, **how)  # from the default stream: waits both ways
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = plan.aed_sample(z, u, **how)
    for _ in range(3):
        for x in got:
            x.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first[0], got[0]) and torch.equal(first[1], got[1])
        assert torch.equal(plan.aed_sample(z, u, **how)[0], first[0])


def test_refusals():
    from paper_2503_05931_amd import vocabulary as L

    def refused(status, f, *a, **kw):
        with pytest.raises(binding.AedError) as e:
            f(*a, **kw)
        assert e.value.status == status and len(str(e.value)) > 12, str(e.value)

    E = binding.AED_EINVAL
    z, u = rows(4, 40)
    z, u = z.cuda(), u.cuda()
    plan = L.Sampler(40, torch.float32)
    f = plan.aed_sample
    refused(E, f, z.bfloat16(), u)
    refused(E, f, z[:, :39], u)
    refused(E, f, z[0], u)
    refused(E, f, z.cpu(), u)
    refused(E, f, z.t().contiguous().t(), u)
    refused(E, f, z[:1].expand(4, 40), u)
    refused(E, f, z, u[:3])
    refused(E, f, z, u.double())
    for kw in (dict(temperature=-1.0), dict(temperature=math.inf), dict(temperature=math.nan), dict(top_k=-1), dict(top_p=1.5), dict(top_p=-0.1), dict(top_p=math.nan),
               dict(min_p=2.0), dict(min_p=-1.0), dict(temperature=u[:2]), dict(top_k=u), dict(top_p=u.cpu()), dict(min_p=u.double())):
        refused(E, f, z, u, **kw)
    tokens, logp = f(z[:0], u[:0])
    assert tokens.shape == logp.shape == (0,)
    refused(binding.AED_EUNSUPPORTED, L.Sampler, 40, torch.float16)
    refused(binding.AED_EUNSUPPORTED, L.Sampler, (1 << 18) + 1, torch.float32)
    plan.close()
    refused(binding.AED_ESTATE, f, z, u)
