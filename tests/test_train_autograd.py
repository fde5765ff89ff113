"""The autograd forms of the training operators (training.Attention.attend, training.Preference.loss) around plans that compute on the host.  No GPU work."""
import pytest
import torch

from paper_2503_05931_amd import training as T


class HostAttention(T.Attention):
    """Calls of a plan, by torch on the host; no library"""

    def __init__(self):
        pass

    def __del__(self):
        pass

    def aed_attn_forward(self, q, k, v, bias=None, key_mask=None):
        s = torch.einsum("ihd,jhd->ihj", q, k)
        return torch.einsum("ihj,jhd->ihd", torch.softmax(s, -1), v), torch.logsumexp(s, -1)

    def aed_attn_backward(self, d_out, q, k, v, out, lse, bias=None, key_mask=None):
        with torch.enable_grad():
            leaves = [t.detach().requires_grad_(True) for t in (q, k, v)]
            return (*torch.autograd.grad(self.aed_attn_forward(*leaves)[0], leaves, d_out.detach()), None)


class HostPreference(T.Preference):
    def __init__(self):
        pass

    def __del__(self):
        pass

    def aed_preference_forward(self, logits, labels, ref):
        gain = torch.log_softmax(logits, 1).gather(1, labels.long()[:, None])[:, 0] - ref
        x = gain[0] - gain[1]
        return -torch.nn.functional.logsigmoid(x), gain, torch.zeros(2, 2)

    def aed_preference_backward(self, logits, labels, ratio, lse, d_loss=None, d_logits=None):
        with torch.enable_grad():
            leaf = logits.detach().requires_grad_(True)
            return torch.autograd.grad(self.aed_preference_forward(leaf, labels, torch.zeros(2))[0], leaf, d_loss.detach())[0]


def attention(cost):
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(3, 2, 64, generator=g).requires_grad_(True) for _ in range(3))
    return cost(HostAttention().attend(q, k, v)), q


def squares():
    return attention(lambda out: out.square().sum())


def row():  # the incoming gradient is a constant
    return attention(lambda out: out[0].sum())


def preference():
    z = torch.randn(2, 5, generator=torch.Generator().manual_seed(0)).requires_grad_(True)
    return HostPreference().loss(z, torch.tensor([1, 2], dtype=torch.int32), torch.zeros(2)), z


@pytest.mark.filterwarnings("ignore:Using backward")
@pytest.mark.parametrize("form", [squares, row, preference])
def test_second_derivatives_are_refused(form):
    """Gradients are made by the library: a term made of them has no gradient of its own, and says so."""
    loss, x = form()
    (plain,) = torch.autograd.grad(loss, x, retain_graph=True)
    assert plain.abs().sum() > 0
    (g,) = torch.autograd.grad(loss, x, create_graph=True)
    assert torch.equal(g, plain)
    loss.backward(retain_graph=True, create_graph=True)  # a graph that nobody goes back through is no mistake
    with pytest.raises(RuntimeError, match="second derivatives"):
        (loss + g.square().sum()).backward()
