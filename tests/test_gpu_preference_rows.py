"""The preference loss in the forms that its launches choose between: rows of one, three and eight vectors a lane, pairs added up by the rows' last workgroup
or by a launch of their own."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def plain(z, labels, ref, lens, beta):
    """(loss, ratio) in float64"""
    lp = torch.log_softmax(z.double(), 1).gather(1, labels.long().clamp(min=0)[:, None])[:, 0] - ref.double()
    gain = torch.where(labels >= 0, lp, torch.zeros_like(lp))
    ratio = torch.stack([part.sum() for part in gain.split(list(lens))])
    return -torch.nn.functional.logsigmoid(beta * (ratio[0::2] - ratio[1::2])).mean(), ratio


# rows up to and above 1600, pairs up to and above 16, logits up to and above 2^23; in float32 a vector has 4, in bfloat16 8
CASES = [([3, 5], 130), ([100] * 16, 512), ([101, 100] + [100] * 14, 512), ([20] * 32, 700), ([20] * 34, 1500), ([0, 1, 7, 0], 4097), ([64, 50], 33000), ([70] * 4, 33000)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lens,vocab", CASES, ids=lambda x: str(x) if isinstance(x, int) else f"{len(x)}x{x[0]}")
def test_forms(lens, vocab, dtype):
    from paper_2503_05931_amd import training as T
    n = sum(lens)
    g = torch.Generator().manual_seed(vocab + n)
    z = (2 * torch.randn((n, vocab), generator=g)).to(dtype)
    labels = torch.randint(0, vocab, (n,), generator=g, dtype=torch.int32)
    labels[::9] = -1
    ref = torch.log_softmax(z.float(), 1).gather(1, labels.long().clamp(min=0)[:, None])[:, 0] + 0.3 * torch.randn(n, generator=g)
    plan = T.Preference(lens, vocab, dtype, beta=0.2)
    args = (z.cuda(), labels.cuda(), ref.cuda())
    leaf = z.double().requires_grad_(True)
    want, want_ratio = plain(leaf, labels, ref, lens, 0.2)
    want.backward()
    first = None
    for _ in range(4):  # the count of arrivals is 0 again after each call
        loss, ratio, lse = plan.aed_preference_forward(*args)
        # a row's terms are of size 2^5 at the most and rounded to 2^-24 of that a few times, a ratio adds up a sequence's
        assert (ratio.cpu().double() - want_ratio.detach()).abs().max() <= 2 ** -17 * max(1, math.sqrt(max(lens)))
        assert abs(loss.item() - want.item()) <= 2 ** -17 * max(1, math.sqrt(max(lens)))
        first = first or (loss.item(), ratio.cpu())
        assert loss.item() == first[0] and torch.equal(ratio.cpu(), first[1])
        d = plan.aed_preference_backward(args[0], args[1], ratio, lse)
        bound = 2 ** -8 if dtype == torch.bfloat16 else 5e-6
        assert (d.cpu().double() - leaf.grad).norm() <= bound * leaf.grad.norm()
        torch.cuda.synchronize()
