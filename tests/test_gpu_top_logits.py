"""A row's largest logits (aed_top_logits) against the definition in float64: values and ids are the row's own and have to be equal.

rest is the float32 log of a float32 sum.  An exponent (z - base) / T is rounded at 2^-24 of itself twice, and of terms that count it is at most 16: 2e-6
of the sum at most, exp2 itself and the sum's roundings 4e-7 more; log and the last addition are rounded at 2^-24 of the result, twice.
"""
import math

import pytest
import torch

from paper_2503_05931_amd import binding
from tests import vocab_reference as R

pytestmark = pytest.mark.gpu

TYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def check(z, top, dtype, t=1.0):
    from paper_2503_05931_amd import vocabulary as L
    print("case", tuple(z.shape), z.stride(0), top, dtype, t, flush=True)
    device = z.to(TYPE[dtype]).cuda() if z.dtype != TYPE[dtype] or not z.is_cuda else z
    values, ids, rest = L.TopLogits(z.shape[1], top, TYPE[dtype], temperature=t).aed_top_logits(device)
    torch.cuda.synchronize()
    for r, row in enumerate(device.float().cpu().numpy()):
        v, i, other = R.top_logits(row, top, float(torch.tensor(t)))
        assert ids[r].tolist() == i, r
        assert values[r].tolist() == v, r
        got = float(rest[r])
        assert got == other or abs(got - other) <= 2.4e-6 + 2 * 2 ** -24 * abs(other), (r, got, other)
    return values, ids, rest


def rows(n, vocab, seed=0):
    g = torch.Generator().manual_seed(seed)
    z = 2 * torch.randn((n, vocab), generator=g)
    return z.scatter_add_(1, torch.randint(0, vocab, (n, 6), generator=g), 10 * torch.rand((n, 6), generator=g))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 5, 63, 64, 128, 255, 256, 257, 300, 511, 513, 1000, 2048, 4096, 4097, 8192, 8200])
def test_vocabularies(vocab, dtype):
    for top in sorted({min(vocab, k) for k in (1, 2, 31, 64, 65, 128)}):
        check(rows(3, vocab, seed=vocab + top), top, dtype, t=2.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [16385, 32768, 33001, 65541, 262144])
def test_wide_vocabularies(vocab, dtype):
    for top in (1, 64, 128):
        check(rows(1, vocab, seed=vocab + top), top, dtype)


def test_same_bits_where_a_wavefront_knows_little():
    """A quarter of a row's lanes hold small logits only, so far more are listed than there is room for, in another order each time."""
    from paper_2503_05931_amd import vocabulary as L
    g = torch.Generator().manual_seed(21)
    z = torch.randn((40, 16384), generator=g)
    z.view(40, 16, 4, 256)[:, :, 3] -= 10                     # every fourth wavefront's vectors
    for top in (2, 4, 8):
        z_d = z.cuda()
        plan = L.TopLogits(16384, top, torch.float32, temperature=3.0)
        first = plan.aed_top_logits(z_d)
        for _ in range(30):
            assert all(torch.equal(a, b) for a, b in zip(plan.aed_top_logits(z_d), first))
        check(z[:8], top, "fp32", t=3.0)


@pytest.mark.parametrize("dtype,vocab", [("fp32", 40003), ("bf16", 70001)])
def test_many_wide_rows(vocab, dtype):
    """More rows than have sixteen wavefronts each: as the definition says, and lists as with a few rows at a time (what is summed, in another order)."""
    from paper_2503_05931_amd import vocabulary as L
    z = rows(258, vocab, seed=9).to(TYPE[dtype])
    z[1], z[2, 100:] = 0.5, -math.inf
    z[3, ::2], z[4] = math.nan, -math.inf
    for top in (8, 128):
        plan = L.TopLogits(vocab, top, TYPE[dtype], temperature=2.0)
        values, ids, rest = plan.aed_top_logits(z.cuda())
        parts = [plan.aed_top_logits(z[i:i + 129].cuda()) for i in (0, 129)]
        assert torch.equal(values, torch.cat([p[0] for p in parts])) and torch.equal(ids, torch.cat([p[1] for p in parts]))
        other = torch.cat([p[2] for p in parts])
        assert torch.equal(rest.isinf(), other.isinf())
        assert ((rest - other).abs()[~rest.isinf()] <= 2 * (2.4e-6 + 2 ** -23 * other.abs()[~rest.isinf()])).all()
        for r in range(6):
            v, i, o = R.top_logits(z[r].float().numpy(), top, 2.0)
            assert ids[r].tolist() == i and values[r].tolist() == v
            assert float(rest[r]) == o or abs(float(rest[r]) - o) <= 2.4e-6 + 2 * 2 ** -24 * abs(o)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [100, 2048, 5000, 33000])
def test_equal_logits(vocab, dtype):
    """The list ends inside of equal ones: it has the lowest ids."""
    at = torch.arange(vocab)
    for z in (torch.full((1, vocab), -2.25), (at % 2).float()[None], -(at % 3).float()[None], torch.where(at % 40 == 7, 5.0, 0.5)[None]):
        for top in (1, 16, 100):
            check(z, top, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [600, 4096])
def test_rows_that_lack_logits(vocab, dtype):
    z = rows(14, vocab, seed=5).to(TYPE[dtype])
    out = torch.rand(z.shape, generator=torch.Generator().manual_seed(6)) < 0.97
    z[0:2][out[0:2]] = -math.inf
    z[2:4][out[2:4]] = math.nan
    z[4:6][out[4:6]] = torch.finfo(TYPE[dtype]).min
    z[6] = -math.inf
    z[7] = math.nan
    z[8] = -math.inf
    z[8, 31:60] = -3.0
    z[9] = torch.finfo(TYPE[dtype]).min
    z[10, 17] = math.inf
    z[11, 17:400] = math.inf
    z[12] = -math.inf
    z[12, 3:35] = 2.0
    z[13, ::2] = -0.0
    z[13, 1::2] = 0.0
    for top in (1, 32, 128):
        check(z, top, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 64, 500, 4000, 16000, 30000, 70001])
def test_rows_with_nothing_in_the_order(vocab, dtype):
    """Every number of wavefronts; rows that have logits between them."""
    z = rows(6, vocab, seed=vocab).to(TYPE[dtype])
    z[0] = z[2] = z[5] = -math.inf
    z[2, ::2] = z[3] = math.nan
    for top in sorted({min(vocab, k) for k in (1, 20, 128)}):
        values, ids, rest = check(z, top, dtype)
        for r in (0, 2, 3, 5):
            assert (values[r] == -math.inf).all() and (ids[r] == -1).all() and float(rest[r]) == -math.inf


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [2048, 4096, 8192, 30000, 70001])
def test_rows_of_nan_at_high_temperatures(vocab, dtype):
    """More NaN than a list holds and nothing in the order, where exponents relative to the list's end are finite: whether such a row is searched is the count's
    decision alone."""
    from paper_2503_05931_amd import vocabulary as L
    z = rows(8, vocab, seed=vocab).to(TYPE[dtype])
    z[0] = z[4] = math.nan
    z[1], z[1, 7::3] = -math.inf, math.nan
    z[2, ::2], z[2, 1::2] = math.nan, -math.nan
    z[3], z[3, :vocab // 2] = -math.inf, math.nan
    z[5, 1:] = math.nan
    for t in (60.0, 100.0, 1e4):
        for top in (1, 32, 128):
            check(z, top, dtype, t=t)
    many = z[[0, 1, 2, 3]].repeat(80, 1).cuda()
    values, ids, rest = L.TopLogits(vocab, 32, TYPE[dtype], temperature=100.0).aed_top_logits(many)
    assert (values == -math.inf).all() and (ids == -1).all() and (rest == -math.inf).all()


@pytest.mark.parametrize("t", [1e-3, 0.05, 30.0, 1e4])
def test_temperatures(t):
    """What is left lies far below the list, or all weights are alike."""
    z = rows(4, 4096, seed=8)
    z[2] *= 100
    z[3, :16] += 3000.0
    for top in (16, 128):
        check(z, top, "fp32", t=t)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("size,t", [(1e-20, 1.0), (1e-31, 1.0), (1e-33, 1.0), (1e-36, 1.0), (1e-39, 1.0), (1e-12, 1e20), (1e-16, 1e20), (1e-25, 1e20), (1.0, 1e20), (1.0, 1e-20),
                                    (1e-19, 1e-20)])
@pytest.mark.parametrize("vocab", [300, 2048, 16384, 70001])
def test_tiny_differences(vocab, size, t, dtype):
    """Exponents that lie by 2^-60 to 2^-130 from each other, and the ends of the temperature's range: what is not listed counts 1 each, or next to nothing."""
    z = (size * rows(2, vocab, seed=vocab).double()).float()
    for top in (1, 16, 128):
        check(z, top, dtype, t=t)


@pytest.mark.parametrize("fill", [-3e4, -1e9, -7e19, -3e37, 2e9])
def test_others_at_one_large_value(fill):
    """Masks of many sizes, few enough of them to be listed, where a list reaches into them and where it does not."""
    z = rows(6, 190, seed=12)
    out = torch.rand((6, 190), generator=torch.Generator().manual_seed(3)) < 0.9
    z[:4][out[:4]] = fill
    z[4] = fill
    z[5] = fill * (1 + torch.arange(190) / 64)
    for top in (4, 40):
        check(z, top, "fp32", t=1.0)
        check(z, top, "fp32", t=0.3)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pitch,skip", [(1024, 0), (1003, 1), (1005, 2), (2000, 3)])
def test_row_strides(pitch, skip, dtype):
    flat = torch.full((9 * pitch + skip,), 100.0, dtype=TYPE[dtype])
    flat.as_strided((9, 1001), (pitch, 1), skip).copy_(rows(9, 1001, seed=pitch))
    device = flat.cuda()
    check(device.as_strided((9, 1001), (pitch, 1), skip), 20, dtype)
    assert torch.equal(device.cpu(), flat)


def test_offsets_past_32_bits():
    far = torch.empty(3 * (1 << 30), dtype=torch.bfloat16, device="cuda").as_strided((3, 900), (1 << 30, 1))
    far.copy_(rows(3, 900, seed=21))
    check(far, 33, "bf16")


@pytest.mark.parametrize("vocab,top", [(4096, 32), (33000, 64)])
def test_same_bits_in_a_graph_and_on_another_stream(vocab, top):
    from paper_2503_05931_amd import vocabulary as L
    z = rows(40, vocab, seed=31).bfloat16().cuda()
    first = L.TopLogits(vocab, top, torch.bfloat16).aed_top_logits(z)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        plan = L.TopLogits(vocab, top, torch.bfloat16)
    again = plan.aed_top_logits(z)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = plan.aed_top_logits(z)
    for _ in range(3):
        for x in got:
            x.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, got))
        assert torch.equal(plan.aed_top_logits(z)[0], first[0])


def test_refusals():
    from paper_2503_05931_amd import vocabulary as L

    def refused(status, f, *a, **kw):
        with pytest.raises(binding.AedError) as e:
            f(*a, **kw)
        assert e.value.status == status and len(str(e.value)) > 12, str(e.value)

    E, U = binding.AED_EINVAL, binding.AED_EUNSUPPORTED
    z = rows(4, 200).cuda()
    plan = L.TopLogits(200, 10, torch.float32)
    f = plan.aed_top_logits
    for bad in (z.bfloat16(), z[:, :199], z[0], z.cpu(), z.t().contiguous().t(), z[:1].expand(4, 200)):
        refused(E, f, bad)
    values, ids, rest = f(z[:0])
    assert values.shape == ids.shape == (0, 10) and rest.shape == (0,)
    refused(E, L.TopLogits, 200, 0, torch.float32)
    refused(E, L.TopLogits, 20, 21, torch.float32)
    refused(U, L.TopLogits, 200, 129, torch.float32)
    refused(E, L.TopLogits, 200, 10, torch.float32, temperature=0.0)
    refused(E, L.TopLogits, 200, 10, torch.float32, temperature=math.nan)
    refused(E, L.TopLogits, 0, 1, torch.float32)
    refused(U, L.TopLogits, (1 << 18) + 1, 10, torch.float32)
    plan.close()
    refused(binding.AED_ESTATE, f, z)
