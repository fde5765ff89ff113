"""The preference loss (aed_preference_forward, aed_preference_backward) against its definition in float64.

Bounds.  A log-probability is a difference of numbers of size 10 or less that are rounded at 2^-24: 1e-6 absolute, and a ratio
of n of them sqrt(n) as much; beta brings that to the loss.  A gradient is slope times a probability, both float32: 1e-6 of
it for the exponent's rounding and what the loss's argument is off; in bfloat16 one rounding more, 2^-8 at most.
"""
import math

import pytest
import torch

from paper_2503_05931_amd import binding
from tests import train_reference as R

pytestmark = pytest.mark.gpu

TYPE = {"fp32": torch.float32, "bf16": torch.bfloat16}


def make(seq_lens, vocab, dtype, seed=0, pitch=0):
    g = torch.Generator().manual_seed(seed)
    rows = sum(seq_lens)
    z = torch.zeros((rows, pitch or vocab), dtype=TYPE[dtype])
    z[:, :vocab] = 2 * torch.randn((rows, vocab), generator=g)
    labels = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    labels[torch.rand(rows, generator=g) < 0.1] = -1
    ref = torch.log_softmax(z[:, :vocab].float(), 1).gather(1, labels.clamp(min=0).long()[:, None])[:, 0] + 0.3 * torch.randn(rows, generator=g)
    return z, labels, ref


def check(z, labels, ref, seq_lens, vocab, dtype, beta=0.1, smoothing=0.0, d_loss=None, place=None):
    from paper_2503_05931_amd import training as T
    print("case", list(seq_lens)[:6], vocab, z.stride(0), dtype, beta, smoothing, flush=True)
    plan = T.Preference(seq_lens, vocab, TYPE[dtype], beta=beta, label_smoothing=smoothing)
    dz, dy, dr = z.cuda(), labels.cuda(), ref.cuda()
    logits = dz[:, :vocab]
    loss, ratio, lse = plan.aed_preference_forward(logits, dy, dr)
    up = None if d_loss is None else torch.tensor(d_loss, dtype=torch.float32, device="cuda")
    grad = plan.aed_preference_backward(logits, dy, ratio, lse, d_loss=up, d_logits=None if place is None else place(dz))
    torch.cuda.synchronize()
    leaf = z[:, :vocab].double().requires_grad_(True)
    want, want_ratio = R.preference(leaf, labels, ref.double(), seq_lens, beta, smoothing)
    (g,) = torch.autograd.grad(want * (1 if d_loss is None else d_loss), leaf, allow_unused=True) if want.requires_grad else (None,)
    g = torch.zeros_like(leaf) if g is None else g
    n = max(1, max(seq_lens))
    assert float((ratio.double().cpu() - want_ratio.detach()).abs().max()) <= 2e-6 * math.sqrt(n) * 4
    assert abs(float(loss) - float(want.detach())) <= beta * 2e-6 * math.sqrt(n) * 4 + 1e-6 * abs(float(want.detach()))
    norm, element = R.off(grad, g)
    slack = 5e-6 + beta * 8e-6 * math.sqrt(n)
    assert norm <= slack + (2 ** -8 if dtype == "bf16" else 0), norm
    assert element <= 4 * slack + (2 ** -7 if dtype == "bf16" else 0), element
    return plan, (logits, dy, dr), (loss, ratio, lse, grad)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 63, 512, 4096, 4097, 9001, 33000])
def test_vocabularies(vocab, dtype):
    lens = [7, 12, 1, 3]
    check(*make(lens, vocab, dtype, seed=vocab), lens, vocab, dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("lens", [[1, 1], [0, 5], [0, 0], [300, 2, 0, 65, 64, 63], [3] * 80], ids=str)
@pytest.mark.parametrize("beta,smoothing,d_loss", [(0.1, 0.0, None), (2.0, 0.1, -3.5)])
def test_lengths(lens, beta, smoothing, d_loss, dtype):
    check(*make(lens, 130, dtype, seed=len(lens)), lens, 130, dtype, beta, smoothing, d_loss)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("pitch", [1024, 1003, 1005])
def test_row_strides_and_gradients_in_place(pitch, dtype):
    """Rows at every alignment, gradients packed, in the logits' place, and in rows that lie otherwise."""
    lens, vocab = [9, 14, 20, 6], 1001
    z, labels, ref = make(lens, vocab, dtype, seed=pitch, pitch=pitch)
    a = check(z, labels, ref, lens, vocab, dtype)[2][3]
    b = check(z, labels, ref, lens, vocab, dtype, place=lambda dz: dz[:, :vocab])[2][3]
    other = torch.full((sum(lens), 1010), 5.0, dtype=TYPE[dtype], device="cuda")
    c = check(z, labels, ref, lens, vocab, dtype, place=lambda dz: other[:, 3:3 + vocab])[2][3]
    assert torch.equal(a, b) and torch.equal(a, c)
    assert (other[:, :3] == 5).all() and (other[:, 3 + vocab:] == 5).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_banned_ids_and_large_logits(dtype):
    """Ids with logit -inf or the type's lowest value, one logit far above the others, labels outside the vocabulary."""
    lens, vocab = [6, 6], 515
    z, labels, ref = make(lens, vocab, dtype, seed=3)
    keep = labels.clamp(min=0).long()
    banned = torch.rand(z.shape, generator=torch.Generator().manual_seed(4)) < 0.3
    banned[torch.arange(12), keep] = False
    z[:6][banned[:6]] = -math.inf
    z[6:][banned[6:]] = torch.finfo(TYPE[dtype]).min
    z[3, keep[3]] = 3000.0
    labels[5], labels[8] = vocab, -7
    check(z, labels, ref.clamp(min=-30), lens, vocab, dtype)
    # a row without a label may hold anything
    labels[4] = -1
    z[4] = float("nan")
    from paper_2503_05931_amd import training as T
    plan = T.Preference(lens, vocab, TYPE[dtype])
    loss, ratio, lse = plan.aed_preference_forward(z.cuda(), labels.cuda(), ref.clamp(min=-30).cuda())
    grad = plan.aed_preference_backward(z.cuda(), labels.cuda(), ratio, lse)
    assert torch.isfinite(loss) and torch.isfinite(grad).all() and not grad[4].any() and not lse[4].any()


def test_gradient_against_differences():
    lens, vocab = [11, 7, 5, 20], 33
    z, labels, ref = make(lens, vocab, "fp32", seed=5)
    grad = check(z, labels, ref, lens, vocab, "fp32", beta=0.5, smoothing=0.05)[2][3].double().cpu()
    u = torch.randn(z.shape, generator=torch.Generator().manual_seed(6)).double()
    f = lambda t: float(R.preference(z.double() + t * u, labels, ref.double(), lens, 0.5, 0.05)[0])
    want = (f(1e-5) - f(-1e-5)) / 2e-5
    assert abs(float((grad * u).sum()) - want) <= 1e-5 * (abs(want) + float(grad.norm()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_same_bits_in_a_graph_and_autograd(dtype):
    from paper_2503_05931_amd import training as T
    lens, vocab = [40, 33, 2, 90], 4096
    _, (z, y, r), first = check(*make(lens, vocab, dtype, seed=7), lens, vocab, dtype)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        plan = T.Preference(lens, vocab, TYPE[dtype])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = plan.aed_preference_forward(z, y, r)
        got += (plan.aed_preference_backward(z, y, got[1], got[2]),)
    for _ in range(3):
        for t in got:
            t.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    leaf = z.clone().requires_grad_(True)
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        (2 * plan.loss(leaf, y, r)).backward()
    torch.cuda.synchronize()
    assert R.off(leaf.grad, 2 * first[3].double())[0] <= 1e-6


def test_refusals():
    from paper_2503_05931_amd import training as T

    def refused(status, f, *a, **kw):
        with pytest.raises(binding.AedError) as e:
            f(*a, **kw)
        assert e.value.status == status and len(str(e.value)) > 12, str(e.value)

    E = binding.AED_EINVAL
    lens, vocab = [3, 4], 40
    z, y, r = (t.cuda() for t in make(lens, vocab, "bf16"))
    plan = T.Preference(lens, vocab, torch.bfloat16)
    refused(E, plan.aed_preference_forward, z.float(), y, r)
    refused(E, plan.aed_preference_forward, z[:, :39], y, r)
    refused(E, plan.aed_preference_forward, z[:6], y, r)
    refused(E, plan.aed_preference_forward, z.t().contiguous().t(), y, r)
    refused(E, plan.aed_preference_forward, z, y.long(), r)
    refused(E, plan.aed_preference_forward, z, y, r[:6])
    refused(E, plan.aed_preference_forward, z.cpu(), y, r)
    refused(E, plan.aed_preference_forward, z[:1].expand(7, vocab), y, r)  # a row stride of 0
    plan.close()
    refused(binding.AED_ESTATE, plan.aed_preference_forward, z, y, r)
