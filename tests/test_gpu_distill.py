"""Distillation (aed_distill_forward, aed_distill_backward) against its definition in float64.

Bounds.  A student's sum of exponentials is float32: exponents rounded twice at 2^-24 of themselves, 16 at most where they count, so 2e-6 of the sum at the
very most, roundings of single terms average out to far less; a row's loss is T^2 times differences of its log to float64 numbers, so 2.5e-6 T^2 absolute, and a
rounding of 2^-24.  Gradients: p has the sum's error and its exponent's, 4e-6 of p together; in the list what is left of p - q is float64, with p from
exact exponents over that sum; with a rest of its own p's multiple outside of the list has the error of both of its terms.  The stored gradient is rounded by half a step
of its type, and once more at 2^-24 through the stored list.
"""
import math

import pytest
import torch

from paper_2503_05931_amd import binding
from tests import vocab_reference as R

pytestmark = pytest.mark.gpu

TYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def make(n, vocab, top, dtype, t=1.0, rest=True, seed=0, unscored=0.2):
    g = torch.Generator().manual_seed(seed)
    teacher = 2 * torch.randn((n, vocab), generator=g)
    teacher.scatter_add_(1, torch.randint(0, vocab, (n, 4), generator=g), 8 * torch.rand((n, 4), generator=g))
    student = (0.9 * teacher + torch.randn((n, vocab), generator=g)).to(TYPE[dtype])
    values, ids, rests = zip(*(R.top_logits(row.numpy(), top, t) for row in teacher))
    weights = torch.rand(n, generator=g) * (torch.rand(n, generator=g) >= unscored)
    return dict(z=student, values=torch.tensor(values, dtype=torch.float32), ids=torch.tensor(ids, dtype=torch.int32),
                rest=torch.tensor(rests, dtype=torch.float32) if rest else None, weights=weights)


def check(c, dtype, t=1.0, d_loss=None, place=None, z_device=None):
    from paper_2503_05931_amd import vocabulary as L
    z, values, ids, rest, weights = (c[n] for n in ("z", "values", "ids", "rest", "weights"))
    n, vocab = z.shape
    top = values.shape[1]
    print("case", n, vocab, top, dtype, t, rest is not None, weights is not None, flush=True)
    plan = L.Distillation(vocab, top, TYPE[dtype], temperature=t)
    on = lambda x: None if x is None else x.cuda()  # noqa: E731
    dz, dv, di, dr, dw = (z.cuda() if z_device is None else z_device), on(values), on(ids), on(rest), on(weights)
    loss, row_loss, stats = plan.aed_distill_forward(dz, dv, di, rest=dr, weights=dw)
    up = None if d_loss is None else torch.tensor(d_loss, dtype=torch.float32, device="cuda")
    grad = plan.aed_distill_backward(dz, di, stats, weights=dw, d_loss=up, d_logits=None if place is None else place(dz))
    torch.cuda.synchronize()
    t = float(torch.tensor(t))  # as the library has it
    want, want_rows = R.distill(z.double(), values, ids, rest, weights, t)
    got = row_loss.double().cpu()
    fine = torch.isfinite(want_rows)
    assert torch.equal(fine, torch.isfinite(got)), (got, want_rows)
    assert torch.equal(got[~fine], want_rows[~fine])
    slack = 2.5e-6 * t * t
    assert ((got - want_rows)[fine].abs() <= slack + 2 ** -22 * want_rows[fine].abs()).all(), ((got - want_rows)[fine].abs().max(), slack)
    if bool(fine.all()):
        weight = 1.0 if weights is None else float(weights.abs().sum())
        assert abs(float(loss) - float(want)) <= slack * weight + 2 ** -22 * abs(float(want)) + 1e-12
    g = R.distill_gradient(z, values, ids, rest, weights, t) * (1 if d_loss is None else d_loss)
    # what p and q are made of, each to 4e-6 of itself
    size = (torch.full((n,), 1 / n) if weights is None else weights).double().abs()[:, None] * t * abs(1 if d_loss is None else d_loss)
    zd = z.double() / t
    p = torch.where(size > 0, torch.nan_to_num(torch.softmax(zd, 1)), 0.0)
    bound = 4e-6 * (g.abs() + 2 * size * p) + (torch.finfo(TYPE[dtype]).eps / 2 + 2 ** -22) * g.abs() + 1e-38
    off = (grad.double().cpu() - g).abs()
    assert (off <= bound).all(), (float((off / bound).max()), int((off > bound).sum()))
    return plan, (dz, dv, di, dr, dw), (loss, row_loss, stats, grad)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 9, 63, 64, 255, 257, 511, 513, 1000, 4096, 4097, 9001])
def test_vocabularies(vocab, dtype):
    for i, (top, rest) in enumerate(((1, True), (8, True), (8, False), (65, True), (128, False))):
        t = (1.0, 2.0, 0.5)[i % 3]
        check(make(4, vocab, min(top, vocab), dtype, t=t, rest=rest, seed=vocab + i), dtype, t=t)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [32768, 33001, 131073, 262144])
def test_wide_vocabularies(vocab, dtype):
    for rest in (True, False):
        check(make(2, vocab, 64, dtype, t=2.0, rest=rest, seed=vocab, unscored=0), dtype, t=2.0)


@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("n", [1, 2, 65, 700])
def test_rows_and_weights(n, rest):
    c = make(n, 130, 5, "bf16", rest=rest, seed=n)
    check(c, "bf16")
    check(c | dict(weights=None), "bf16", d_loss=-3.5)
    c["weights"][0] = -2.0
    check(c, "bf16", d_loss=0.25)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [True, False])
def test_lists(rest, dtype):
    """Ids twice and three times, entries that are left out, lists with nothing, longer than the vocabulary, of the whole vocabulary."""
    c = make(8, 300, 12, dtype, rest=rest, seed=2, unscored=0)
    ids, values = c["ids"], c["values"]
    ids[0, 3] = ids[0, 7]
    ids[1, 1] = ids[1, 4] = ids[1, 11]
    ids[2, 2:] = -1
    ids[3, :4] = torch.tensor([300, -5, 2 ** 31 - 1, -2 ** 31])
    values[4, 3:6] = -math.inf
    ids[5] = -1
    values[6] = -math.inf
    if rest:
        c["rest"][5] = -math.inf
        c["rest"][7] = -math.inf
    check(c, dtype)
    for vocab in (4, 20):
        c = make(5, vocab, vocab, dtype, rest=rest, seed=vocab, unscored=0)
        more = 128 - vocab
        c["ids"] = torch.cat((c["ids"], torch.randint(0, vocab, (5, more), dtype=torch.int32, generator=torch.Generator().manual_seed(1))), 1)
        c["values"] = torch.cat((c["values"], torch.full((5, more), -1.0)), 1)
        check(c, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_unscored_rows_hold_anything(dtype):
    c = make(6, 200, 7, dtype, seed=3, unscored=0)
    c["weights"][2] = c["weights"][4] = 0.0
    c["z"][2], c["z"][4] = math.nan, -math.inf
    c["values"][2], c["ids"][4], c["rest"][2] = math.nan, 5000, math.nan
    loss, row_loss, _, grad = check(c, dtype)[2]
    assert torch.isfinite(loss) and not row_loss[[2, 4]].any() and not grad[[2, 4]].any() and torch.isfinite(grad).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("vocab", [90, 4097, 20001])
def test_rows_with_neither_an_entry_nor_a_rest(vocab, rest, dtype):
    """Their loss and gradient are 0, whatever their logits hold."""
    from paper_2503_05931_amd import vocabulary as L
    c = make(7, vocab, 5, dtype, t=0.25, rest=rest, seed=vocab, unscored=0)
    c["ids"][:3] = -1
    c["values"][3:6] = -math.inf
    if rest:
        c["rest"][:6] = -math.inf
    for i, fill in enumerate((200.0, math.nan, math.inf, torch.finfo(TYPE[dtype]).max, -math.inf)):
        c["z"][i] = fill
    for weights in (c["weights"], None):
        _, (z, _, ids, _, w), (loss, row_loss, stats, grad) = check(c | dict(weights=weights), dtype, t=0.25)
        assert not grad[:6].any() and not row_loss[:6].any() and grad[6].any() and torch.isfinite(loss)
        place = L.Distillation(vocab, 5, TYPE[dtype], temperature=0.25).aed_distill_backward(z, ids, stats, weights=w, d_logits=z)
        assert place is z and torch.equal(place, grad)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("vocab,top", [(300, 6), (300, 70), (20001, 6)])
def test_teachers_that_are_not_numbers(vocab, top, rest, dtype):
    """Entries that are NaN or infinite make their row's loss NaN, and its gradient by their ids, also where the list has no others; a rest that is neither
    counts as none where there is no entry.  Other rows are as they would be without them."""
    from paper_2503_05931_amd import vocabulary as L
    c = make(9, vocab, top, dtype, rest=rest, seed=vocab + top, unscored=0)
    c["values"][0] = math.nan
    c["values"][1, 3] = math.nan
    c["values"][2] = math.nan
    c["values"][3], c["ids"][3, 1:] = math.nan, -1
    c["values"][4] = math.inf
    c["ids"][5:8] = -1
    bad, empty = [0, 1, 2, 3, 4], [5, 6, 7]
    if rest:
        c["rest"][2] = c["rest"][3] = -math.inf
        c["rest"][5:8] = torch.tensor([math.inf, math.nan, -math.inf])
    z, ids = c["z"].cuda(), c["ids"].cuda()
    on = dict(values=c["values"].cuda(), ids=ids, rest=c["rest"].cuda() if rest else None)
    plan = L.Distillation(vocab, top, TYPE[dtype])
    loss, rows, stats = plan.aed_distill_forward(z, **on)
    grad = plan.aed_distill_backward(z, ids, stats)
    assert loss.isnan() and rows[bad].isnan().all() and not rows[empty].any() and not grad[empty].any()
    for r in bad:
        assert grad[r][ids[r][ids[r] >= 0].long()].isnan().all(), r
    check({n: None if v is None else v[8:] for n, v in c.items()}, dtype)
    alone = plan.aed_distill_forward(z[8:], **{n: None if v is None else v[8:] for n, v in on.items()})[1]
    assert torch.equal(rows[8:], alone)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("vocab", [90, 4097, 20001])
def test_students_that_are_not_numbers(vocab, rest, dtype):
    """NaN and plus infinity give NaN: the row's loss, and its gradient by the list and by all others that are not minus infinity; also where the row, or what
    is outside of the list, has no number at all."""
    from paper_2503_05931_amd import vocabulary as L
    c = make(7, vocab, 5, dtype, rest=rest, seed=vocab, unscored=0)
    z, ids = c["z"], c["ids"].long()
    keep = torch.gather(z, 1, ids)
    z[0] = math.nan
    z[1], z[1, ::2] = -math.inf, math.nan
    z[2], z[3] = math.nan, math.inf
    z[4, vocab // 2] = math.nan
    z[5, 0] = math.inf
    z[2].scatter_(0, ids[2], keep[2])
    z = z.cuda()
    plan = L.Distillation(vocab, 5, TYPE[dtype])
    loss, rows, stats = plan.aed_distill_forward(z, c["values"].cuda(), c["ids"].cuda(), rest=c["rest"].cuda() if rest else None)
    grad = plan.aed_distill_backward(z, c["ids"].cuda(), stats)
    assert loss.isnan() and rows[:6].isnan().all() and torch.isfinite(rows[6])
    assert (grad[:6].isnan() | (z[:6] == -math.inf)).all() and torch.isfinite(grad[6]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [True, False])
def test_students_without_mass(rest, dtype):
    """Ids that the student excludes, listed and not; a student without any logit; only the list, only others."""
    c = make(6, 250, 9, dtype, rest=rest, seed=4, unscored=0)
    z, ids = c["z"], c["ids"].long()
    z[0, ids[0, 2]] = -math.inf                               # the teacher wants it: infinite
    z[1][torch.rand(250, generator=torch.Generator().manual_seed(5)) < 0.5] = -math.inf
    z[1, ids[1]] = 1.0
    z[2] = -math.inf
    z[3] = -math.inf
    z[3, ids[3]] = 0.5                                        # no others
    z[4, ids[4]] = -math.inf                                  # only others
    z[5] = torch.finfo(TYPE[dtype]).min
    z[5, ids[5]] = 2.0
    check(c, dtype)


@pytest.mark.parametrize("t", [0.25, 1.0, 5.0])
def test_sure_students(t):
    """What the student leaves for others is 1e-9, 1e-30 and 1e-90 of the row: its log and the gradient's ratio keep their digits."""
    c = make(3, 400, 6, "fp32", t=t, seed=6, unscored=0)
    for r, far in enumerate((20.0, 70.0, 210.0)):
        c["z"][r, c["ids"][r].long()] += far * t
    check(c, "fp32", t=t)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab,t", [(700, 3.0), (4096, 5.5), (33001, 7.0), (33001, 3.3)])
def test_small_divergences(vocab, t, dtype):
    """At a high temperature a row's loss is T^2 times a small difference of logarithms.  What all terms of a sum may have in common is the exponential's own
    error, one step of float32, 2^-23, and as much for the additions of a thread; an exponent's roundings have either sign and average out.  So 2.5e-7 T^2, ten
    times less than what is allowed elsewhere; an inverse temperature that were a float alone would add 2^-24 of the mean exponent, some 1e-6 T^2."""
    from paper_2503_05931_amd import vocabulary as L
    g = torch.Generator().manual_seed(vocab)
    c = make(40, vocab, 32, dtype, t=t, seed=vocab, unscored=0)
    c["z"] = (3 * (c["z"].float() - 8)).to(TYPE[dtype])
    c["values"], c["ids"], c["rest"] = (torch.tensor(x) for x in zip(*(R.top_logits(row.numpy(), 32, t) for row in
                                        c["z"].float() + 0.02 * torch.randn(c["z"].shape, generator=g))))
    c["values"], c["ids"], c["rest"] = c["values"].float(), c["ids"].int(), c["rest"].float()
    for name in ("others", "list alone"):
        rest = c["rest"] if name == "others" else None
        _, got, _ = L.Distillation(vocab, 32, TYPE[dtype], temperature=t).aed_distill_forward(
            c["z"].cuda(), c["values"].cuda(), c["ids"].cuda(), rest=None if rest is None else rest.cuda(), weights=None)
        want = R.distill(c["z"].double(), c["values"], c["ids"], rest, None, float(torch.tensor(t)))[1]
        assert (got.double().cpu() - want).abs().max() <= 2.5e-7 * t * t + 2 ** -22 * float(want.abs().max()), name


@pytest.mark.parametrize("fill", [-3e4, -1e9, -7e19, -3e37])
def test_others_at_one_low_value(fill):
    """Masks of many sizes: what is outside of the list is all alike, and its mass that of so many ids at the value."""
    c = make(4, 300, 6, "fp32", seed=9, unscored=0)
    keep = torch.gather(c["z"], 1, c["ids"].long())
    c["z"][:] = fill
    check(c, "fp32")
    c["z"].scatter_(1, c["ids"].long(), keep)
    check(c, "fp32")


def test_temperatures_and_large_logits():
    for t in (0.01, 50.0, 1000.0):
        check(make(4, 500, 10, "fp32", t=t, seed=7, unscored=0), "fp32", t=t)
    c = make(4, 500, 10, "fp32", seed=8, unscored=0)
    c["z"] = c["z"] + 1e4
    c["values"] = c["values"] - 1e4
    c["rest"] = c["rest"] - 1e4
    check(c, "fp32")


def test_gradient_against_differences():
    for rest in (True, False):
        c = make(5, 60, 6, "fp32", t=1.5, rest=rest, seed=9)
        c["ids"][0, 1] = c["ids"][0, 0]
        grad = check(c, "fp32", t=1.5)[2][3].double().cpu()
        u = torch.randn(c["z"].shape, generator=torch.Generator().manual_seed(6)).double()
        f = lambda h: float(R.distill(c["z"].double() + h * u, c["values"], c["ids"], c["rest"], c["weights"], 1.5)[0])  # noqa: E731
        want = (f(1e-5) - f(-1e-5)) / 2e-5
        assert abs(float((grad * u).sum()) - want) <= 1e-5 * (abs(want) + float(grad.norm()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rest", [True, False])
@pytest.mark.parametrize("vocab,pitch,skip", [(1001, 1024, 0), (1001, 1003, 1), (1001, 1005, 2), (5, 9, 3), (20001, 20011, 1)])
def test_row_strides_and_gradients_in_place(vocab, pitch, skip, rest, dtype):
    """Rows at every alignment, gradients packed, in the logits' place, and in rows that lie otherwise; what lies beside is left alone."""
    c = make(6, vocab, min(20, vocab), dtype, rest=rest, seed=pitch)
    flat = torch.full((6 * pitch + 8,), 100.0, dtype=TYPE[dtype], device="cuda")
    view = flat.as_strided((6, vocab), (pitch, 1), skip)
    view.copy_(c["z"])
    a = check(c, dtype, z_device=view)[2][3]
    other = torch.full((6 * (pitch + 5) + 8,), 5.0, dtype=TYPE[dtype], device="cuda")
    to = other.as_strided((6, vocab), (pitch + 5, 1), 1)
    b = check(c, dtype, z_device=view, place=lambda _: to)[2][3]
    assert torch.equal(a, b)
    left = other.clone()
    left.as_strided((6, vocab), (pitch + 5, 1), 1).fill_(5.0)
    assert (left == 5).all()
    b = check(c, dtype, z_device=view, place=lambda dz: dz)[2][3]
    assert torch.equal(a, b)
    view.fill_(100.0)
    assert (flat == 100).all()


def test_gradients_by_other_ids_stay_in_their_rows():
    """ids are looked at again: those that do not belong to the stats reach no other row."""
    from paper_2503_05931_amd import vocabulary as L
    c = make(5, 90, 7, "fp32", seed=14, unscored=0)
    plan = L.Distillation(90, 7, torch.float32)
    z, ids = c["z"].cuda(), c["ids"].cuda()
    stats = plan.aed_distill_forward(z, c["values"].cuda(), ids, rest=c["rest"].cuda())[2]
    ids[0, 1], ids[2, 3], ids[4, 6] = 91, -1, 2 ** 31 - 1
    place = torch.full((5, 100), 7.0, device="cuda")
    plan.aed_distill_backward(z, ids, stats, d_logits=place[:, :90])
    assert (place[:, 90:] == 7).all()


def test_offsets_past_32_bits():
    c = make(3, 900, 9, "bf16", seed=11, unscored=0)
    far = torch.empty(3 * (1 << 30), dtype=torch.bfloat16, device="cuda").as_strided((3, 900), (1 << 30, 1))
    far.copy_(c["z"])
    check(c, "bf16", z_device=far, place=lambda dz: dz)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_same_bits_in_a_graph_and_autograd(dtype):
    from paper_2503_05931_amd import vocabulary as L
    c = make(150, 4096, 32, dtype, t=2.0, seed=12)
    _, given, first = check(c, dtype, t=2.0)
    z, v, i, r, w = given
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        plan = L.Distillation(4096, 32, TYPE[dtype], temperature=2.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        loss, rows, stats = plan.aed_distill_forward(z, v, i, rest=r, weights=w)
        grad = plan.aed_distill_backward(z, i, stats, weights=w)
    for _ in range(3):
        for x in (loss, rows, grad):
            x.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((first[0], first[1], first[3]), (loss, rows, grad)))
        assert torch.equal(plan.aed_distill_forward(z, v, i, rest=r, weights=w)[0], first[0])
    leaf = z.clone().requires_grad_(True)
    loss = 2 * plan.loss(leaf, v, i, rest=r, weights=w)  # from the default stream: waits both ways
    loss.backward()
    torch.cuda.synchronize()
    scale = (leaf.grad.double() - 2 * first[3].double()).norm() / (2 * first[3].double()).norm()
    assert float(scale) <= 1e-6


def test_no_rows():
    from paper_2503_05931_amd import vocabulary as L
    plan = L.Distillation(50, 4, torch.float32)
    z, v, i = torch.empty((0, 50), device="cuda"), torch.empty((0, 4), device="cuda"), torch.empty((0, 4), dtype=torch.int32, device="cuda")
    loss, rows, stats = plan.aed_distill_forward(z, v, i)
    assert float(loss) == 0 and rows.shape == (0,) and plan.aed_distill_backward(z, i, stats).shape == (0, 50)


def test_refusals():
    from paper_2503_05931_amd import vocabulary as L

    def refused(status, f, *a, **kw):
        with pytest.raises(binding.AedError) as e:
            f(*a, **kw)
        assert e.value.status == status and len(str(e.value)) > 12, str(e.value)

    E, U = binding.AED_EINVAL, binding.AED_EUNSUPPORTED
    c = make(5, 40, 6, "fp32", seed=1)
    z, v, i, r, w = (c[n].cuda() for n in ("z", "values", "ids", "rest", "weights"))
    plan = L.Distillation(40, 6, torch.float32)
    f, b = plan.aed_distill_forward, plan.aed_distill_backward
    _, _, stats = f(z, v, i, rest=r, weights=w)
    for bad in (z.bfloat16(), z[:, :39], z[:4], z[0], z.cpu(), z.t().contiguous().t(), z[:1].expand(5, 40)):
        refused(E, f, bad, v, i)
        refused(E, b, bad, i, stats)
    refused(E, f, z, v[:, :5], i)
    refused(E, f, z, v.double(), i)
    refused(E, f, z, v, i.long())
    refused(E, f, z, v, i, rest=r[:4])
    refused(E, f, z, v, i, weights=w.cpu())
    refused(E, b, z, i, stats[:, :7])
    refused(E, b, z, i, stats, weights=w[:2])
    refused(E, b, z, i, stats, d_logits=z[:, :30])
    refused(E, b, z, i, stats, d_loss=torch.ones(1, device="cuda", dtype=torch.float64).reshape(()))
    wide = torch.zeros((5, 80), device="cuda")
    refused(E, b, wide[:, :40], i, stats, d_logits=wide.as_strided((5, 40), (60, 1)))  # in the logits' place, at another distance
    refused(E, L.Distillation, 40, 0, torch.float32)
    refused(U, L.Distillation, 40, 129, torch.float32)
    refused(E, L.Distillation, 40, 6, torch.float32, temperature=-1.0)
    refused(E, L.Distillation, 40, 6, torch.float32, temperature=math.inf)
    refused(U, L.Distillation, (1 << 18) + 1, 6, torch.float32)
    plan.close()
    refused(binding.AED_ESTATE, f, z, v, i)
