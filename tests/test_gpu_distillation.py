"""The operators on rows of logits together, behind the decoder's step, as a server and examples/distillation.py use them."""
import importlib.util
import math
import os

import pytest
import torch

from tests import vocab_reference as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def decoder(**kw):
    from paper_2503_05931_amd import binding, workloads as W
    wl = W.make("tiny")
    dec = binding.Decoder(wl.cfg, wl.weights, max_batch=wl.cfg.batch, max_total_enc_frames=int(wl.enc_lens.sum()), max_dec_len=wl.cfg.max_dec_len, **kw)
    dec.aed_cross_kv_precompute(dec.to_device(wl.enc), wl.enc_lens)
    return wl, dec


def test_sampling_behind_the_decoders_step():
    """Temperature 0 is the decoder's own choice; drawn tokens are those of the definition, step for step, fed back to the decoder."""
    from paper_2503_05931_amd import vocabulary as L
    wl, dec = decoder()
    sampler = L.Sampler(wl.cfg.vocab, torch.float32)
    gen = torch.Generator(device="cuda").manual_seed(3)
    fed = torch.from_numpy(wl.prompt[:, 0].copy()).cuda()
    t = torch.tensor([0.0, 0.8, 1.0, 1.3], device="cuda")[:wl.cfg.batch]
    k = torch.tensor([0, 40, 0, 200], dtype=torch.int32, device="cuda")[:wl.cfg.batch]
    p = torch.tensor([1.0, 0.9, 0.7, 1.0], device="cuda")[:wl.cfg.batch]
    for _ in range(12):
        greedy, logits = dec.aed_decode_step(fed)
        u = torch.rand(wl.cfg.batch, generator=gen, device="cuda")
        none, _ = sampler.aed_sample(logits, u, temperature=0.0)
        assert torch.equal(none, greedy)
        fed, logp = sampler.aed_sample(logits, u, temperature=t, top_k=k, top_p=p)
        for r, z in enumerate(logits.cpu().numpy()):
            token, lp = R.sample(z, float(u[r]), t=float(t[r]), top_k=int(k[r]), top_p=float(p[r]))
            assert int(fed[r]) == token and abs(float(logp[r]) - lp) <= 2 ** -24 * abs(lp) + 1e-9
    dec.close()


def test_a_captured_step_samples_its_next_token():
    """The step that allocates nothing and the sampler behind it on the decoder's stream, captured and replayed: each replay feeds what the one before has drawn."""
    from paper_2503_05931_amd import vocabulary as L
    results = []
    for captured in (False, True):
        stream = torch.cuda.Stream()
        wl, dec = decoder(stream=stream)
        B, V = wl.cfg.batch, wl.cfg.vocab
        with torch.cuda.stream(stream):
            sampler = L.Sampler(V, torch.float32)
            uniforms = torch.rand((10, B), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
            u, fed, out = torch.empty(B, device="cuda"), torch.from_numpy(wl.prompt[:, 0].copy()).cuda(), torch.empty(B, dtype=torch.int32, device="cuda")
            logits = torch.empty((B, V), device="cuda")

            def step():
                dec.aed_decode_step_noalloc(fed, out, logits)
                tokens, logp = sampler.aed_sample(logits, u, temperature=0.9, top_k=50)
                fed.copy_(tokens)
                return tokens, logp

            got = []
            for s in range(10):
                u.copy_(uniforms[s])
                if not captured or s == 0:  # the first step takes pages, which no replay does again
                    tokens, logp = step()
                else:  # the decoder counts positions on the host: a capture is one step
                    graph = torch.cuda.CUDAGraph()
                    torch.cuda.synchronize()
                    with torch.cuda.graph(graph, stream=stream):
                        tokens, logp = step()
                    graph.replay()
                torch.cuda.synchronize()
                got.append((tokens.clone(), logp.clone()))
        results.append(got)
        dec.close()
    for a, b in zip(*results):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("top", [1, 16, 128])
def test_lists_carry_the_teacher(top, dtype):
    """A teacher's rows through aed_top_logits into the loss: the divergence over the list's ids and one class for all others, from the rows themselves.
    A list of the whole vocabulary is the whole divergence.  The lists' float32 rest adds 2^-23 of its logarithm, 12, to the bounds of
    the loss's own tests."""
    from paper_2503_05931_amd import vocabulary as L
    T = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    for vocab in (128, 3001):
        g = torch.Generator().manual_seed(vocab + top)
        teacher = (3 * torch.randn((40, vocab), generator=g)).to(T)
        student = (teacher.float() + torch.randn((40, vocab), generator=g)).to(T)
        t = 2.0
        lists = L.TopLogits(vocab, top, T, temperature=t).aed_top_logits(teacher.cuda())
        plan = L.Distillation(vocab, top, T, temperature=t)
        leaf = student.cuda().requires_grad_(True)
        loss = plan.loss(leaf, *lists)
        loss.backward()
        z = student.double().requires_grad_(True)
        log_q, log_p = torch.log_softmax(teacher.double() / t, 1), torch.log_softmax(z / t, 1)
        ids = torch.sort(teacher.float(), dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(lists[1].cpu().long(), ids)
        rows = (log_q.gather(1, ids).exp() * (log_q.gather(1, ids) - log_p.gather(1, ids))).sum(1)
        if top < vocab:
            others = torch.ones((40, vocab), dtype=torch.bool).scatter(1, ids, False)
            q, p = (torch.where(others, x.exp(), 0.0).sum(1) for x in (log_q, log_p))
            rows = rows + q * (q.log() - p.log())
        want = t * t * rows.mean()
        want.backward()
        loss, want = loss.detach(), want.detach()
        bound = 2.5e-6 * t * t + t * t * 12 * 2 ** -23
        assert abs(float(loss) - float(want)) <= bound + 2 ** -22 * float(want)
        p = torch.softmax(student.double() / t, 1) * t / 40
        off = (leaf.grad.double().cpu() - z.grad).abs()
        assert (off <= (4e-6 + 12 * 2 ** -23) * (z.grad.abs() + 2 * p) + (torch.finfo(T).eps / 2 + 2 ** -22) * z.grad.abs() + 1e-38).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_example(dtype):
    """It runs, its losses are finite, and every parameter has a finite gradient that is not all zero."""
    spec = importlib.util.spec_from_file_location("distillation", os.path.join(ROOT, "examples", "distillation.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    model, tokens, losses = example.main(steps=3, dtype=dtype, say=lambda s: None)
    assert tokens.shape[1] > 20 and int(tokens.min()) >= 0 and len(losses) == 3 and all(math.isfinite(x) and x > 0 for x in losses)
    for name, p in model.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad).all(), name
    assert sum(float(p.grad.float().abs().sum()) > 0 for p in model.parameters()) >= 0.9 * len(list(model.parameters()))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_every_parameter_of_the_example_has_a_gradient(dtype):
    """None is all zeros, without an exception."""
    spec = importlib.util.spec_from_file_location("distillation", os.path.join(ROOT, "examples", "distillation.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    model, _, _ = example.main(steps=1, dtype=dtype, say=lambda s: None)
    assert not [name for name, p in model.named_parameters() if p.grad is None or not p.grad.any()]
