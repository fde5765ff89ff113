"""A smaller decoder learns from what the library's decoder answers.

The teacher (paper_2503_05931_amd.binding.Decoder) transcribes a batch step by step: its tokens are drawn from its logits by temperature, top-k and top-p, and
of every step's logits the largest are kept, with the mass of all others.  The student, a decoder of fewer layers, reads the same transcripts and is trained on
these lists: the divergence of its rows from the teacher's, prompts and all, comes straight from its packed logits.

    python examples/distillation.py [--steps 20] [--dtype fp32|bf16]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paper_2503_05931_amd import binding, vocabulary, workloads as W  # noqa: E402
from preference_tuning import Decoder  # noqa: E402

TOP, TEMPERATURE = 16, 2.0


def transcripts(seed=0, new=24):
    """A batch that the library's decoder has written: the workload, tokens [batch, positions], and the lists of the rows that predict all
    but the first of them, [batch, positions - 1, ...]."""
    wl = W.make("tiny")
    cfg = wl.cfg
    dec = binding.Decoder(cfg, wl.weights, max_batch=cfg.batch, max_total_enc_frames=int(wl.enc_lens.sum()), max_dec_len=cfg.max_dec_len)
    dec.aed_cross_kv_precompute(dec.to_device(wl.enc), wl.enc_lens)
    prompt = torch.from_numpy(wl.prompt).to(dec.device)
    gen = torch.Generator(device=dec.device).manual_seed(seed)
    sampler = vocabulary.Sampler(cfg.vocab, torch.float32)
    teacher = vocabulary.TopLogits(cfg.vocab, TOP, torch.float32, temperature=TEMPERATURE)
    tokens, lists = [prompt[:, 0].contiguous()], []
    for s in range(prompt.shape[1] + new - 1):
        _, logits = dec.aed_decode_step(tokens[-1])
        lists.append(teacher.aed_top_logits(logits))
        if s + 1 < prompt.shape[1]:
            tokens.append(prompt[:, s + 1].contiguous())
        else:
            u = torch.rand(cfg.batch, generator=gen, device=dec.device)
            tokens.append(sampler.aed_sample(logits, u, temperature=0.8, top_k=100, top_p=0.95)[0])
    torch.cuda.synchronize()
    dec.close()
    return wl, torch.stack(tokens, 1), [torch.stack(part, 1) for part in zip(*lists)]


def main(steps=20, dtype="fp32", seed=0, say=print):
    torch.manual_seed(seed)
    wl, tokens, lists = transcripts(seed)
    cfg, dev = wl.cfg, tokens.device
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    model = Decoder(cfg.vocab, cfg.d_model, cfg.n_heads, cfg.d_ffn, layers=1).to(dev, dt)
    n, rows = tokens.shape[0], tokens.shape[1] - 1
    own, cross = model.plans([rows] * n, wl.enc_lens)
    enc = torch.from_numpy(wl.enc).to(dev, dt)
    inputs = tokens[:, :-1].flatten().long()
    values, ids, rest = (t.flatten(0, 1).contiguous() for t in lists)
    # what the prompt itself says is given, and not learned
    scored = torch.arange(rows, device=dev) + 1 >= wl.prompt.shape[1]
    weights = (scored.float() / (n * scored.sum())).repeat(n)
    loss_of = vocabulary.Distillation(cfg.vocab, TOP, dt, temperature=TEMPERATURE)
    opt = torch.optim.Adam(model.parameters(), lr=1e-3)
    losses = []
    for step in range(steps):
        opt.zero_grad()
        loss = loss_of.loss(model(inputs, enc, own, cross), values, ids, rest, weights)
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
        say(f"step {step}: divergence from the teacher {losses[-1]:.4f}")
    return model, tokens, losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    args = ap.parse_args()
    main(args.steps, args.dtype)
