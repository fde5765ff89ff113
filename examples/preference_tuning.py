"""Preference tuning of a small decoder on the mistakes of the library's own decoding.

The greedy decoder transcribes a batch (paper_2503_05931_amd.binding.Decoder); where its transcript differs from the reference
one, the pair (reference preferred, decoded not) is trained on.  The decoder that is tuned attends as the library's does,
with a learned relative position bias in its self-attention: one plan for the self-attention and one for the cross-attention
of a batch serve all layers, forward and backward, and the preference loss comes straight from the packed logits.  At
the end the tuned decoder writes tokens one by one against caches, through the same operators' single-row form.

    python examples/preference_tuning.py [--steps 20] [--dtype fp32|bf16]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2503_05931_amd import binding, training, workloads as W  # noqa: E402

BUCKETS, DISTANCE = 16, 64


class Layer(torch.nn.Module):
    def __init__(self, d, heads, ffn):
        super().__init__()
        self.heads, self.head = heads, d // heads
        self.ln1, self.ln2, self.ln3 = (torch.nn.LayerNorm(d) for _ in range(3))
        self.qkv, self.o = torch.nn.Linear(d, 3 * d), torch.nn.Linear(d, d)
        self.cq, self.ckv, self.co = torch.nn.Linear(d, d), torch.nn.Linear(d, 2 * d), torch.nn.Linear(d, d)
        self.up, self.down = torch.nn.Linear(d, ffn), torch.nn.Linear(ffn, d)
        self.bias = torch.nn.Parameter(0.1 * torch.randn(BUCKETS, heads))

    def split(self, x, parts):
        """[rows, parts * d] -> parts tensors [rows, heads, head], without a copy"""
        return x.view(x.shape[0], parts, self.heads, self.head).unbind(1)

    def forward(self, x, enc, own, cross):
        q, k, v = self.split(self.qkv(self.ln1(x)), 3)
        x = x + self.o(own.attend(q, k, v, bias=self.bias).flatten(1))
        k, v = self.split(self.ckv(enc), 2)
        q, = self.split(self.cq(self.ln2(x)), 1)
        x = x + self.co(cross.attend(q, k, v).flatten(1))
        return x + self.down(torch.relu(self.up(self.ln3(x))))


class Decoder(torch.nn.Module):
    def __init__(self, vocab, d=256, heads=4, ffn=1024, layers=2):
        super().__init__()
        self.d, self.heads, self.head = d, heads, d // heads
        self.emb = torch.nn.Embedding(vocab, d)
        self.layers = torch.nn.ModuleList(Layer(d, heads, ffn) for _ in range(layers))
        self.ln, self.out = torch.nn.LayerNorm(d), torch.nn.Linear(d, vocab)

    def plans(self, lens, enc_lens, **kw):
        """The two plans of a batch: rows of a sequence among themselves, and to its frames"""
        dtype = self.emb.weight.dtype
        return (training.Attention(lens, lens, self.heads, self.head, dtype, causal=True, bias_buckets=BUCKETS, bias_max_distance=DISTANCE, **kw),
                training.Attention(lens, enc_lens, self.heads, self.head, dtype, **kw))

    def forward(self, tokens, enc, own, cross):
        """tokens, enc: packed rows; returns the packed logits"""
        x = self.emb(tokens)
        for layer in self.layers:
            x = layer(x, enc, own, cross)
        return self.out(self.ln(x))

    @torch.no_grad()
    def write(self, first, enc, enc_lens, steps):
        """Greedy decoding, one row a sequence and step, against caches of `steps` positions.  Returns tokens and the steps' logits."""
        n, dtype, dev = len(enc_lens), self.emb.weight.dtype, enc.device
        starts = np.arange(n) * steps
        at = torch.from_numpy(starts).to(dev)
        caches = [torch.zeros((2, n * steps, self.heads, self.head), dtype=dtype, device=dev) for _ in self.layers]
        frames = [layer.split(layer.ckv(enc), 2) for layer in self.layers]
        cross = training.Attention([1] * n, enc_lens, self.heads, self.head, dtype, training=False)
        tokens, logits = [first], []
        for s in range(steps):
            own = training.Attention([1] * n, [s + 1] * n, self.heads, self.head, dtype, causal=True, bias_buckets=BUCKETS,
                                     bias_max_distance=DISTANCE, k_starts=starts, training=False)
            x = self.emb(tokens[-1])
            for layer, (ck, cv), (fk, fv) in zip(self.layers, caches, frames):
                q, k, v = layer.split(layer.qkv(layer.ln1(x)), 3)
                ck[at + s], cv[at + s] = k, v
                x = x + layer.o(own.aed_attn_forward(q, ck, cv, bias=layer.bias)[0].flatten(1))
                q, = layer.split(layer.cq(layer.ln2(x)), 1)
                x = x + layer.co(cross.aed_attn_forward(q, fk, fv)[0].flatten(1))
                x = x + layer.down(torch.relu(layer.up(layer.ln3(x))))
            logits.append(self.out(self.ln(x)))
            tokens.append(logits[-1].argmax(-1))
        return torch.stack(tokens[1:], 1), torch.stack(logits, 1)


def pairs(seed=0):
    """A batch that the library's decoder has transcribed: encoder states, their lengths, and for every utterance the
    preferred and the decoded transcript (with the prompt in front)."""
    wl = W.make("tiny")
    cfg = wl.cfg
    dec = binding.Decoder(cfg, wl.weights, max_batch=cfg.batch, max_total_enc_frames=int(wl.enc_lens.sum()), max_dec_len=cfg.max_dec_len)
    dec.aed_cross_kv_precompute(dec.to_device(wl.enc), wl.enc_lens)
    decoded, _ = dec.aed_greedy_decode(torch.from_numpy(wl.prompt).to(dec.device), cfg.max_new)
    decoded = decoded.cpu().numpy()
    dec.close()
    rng = np.random.default_rng(seed)
    seqs = []
    for prompt, ids in zip(wl.prompt, decoded):  # stands in for human transcripts: other words, another length
        n = int(rng.integers(12, cfg.max_new + 1))
        wanted = rng.integers(3, cfg.vocab, size=n)
        seqs += [np.concatenate([prompt, wanted]), np.concatenate([prompt, ids])]
    return wl, cfg, seqs


def main(steps=20, dtype="fp32", seed=0, say=print):
    torch.manual_seed(seed)
    wl, cfg, seqs = pairs(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    dev, P = torch.device("cuda"), wl.prompt.shape[1]
    model = Decoder(cfg.vocab, cfg.d_model, cfg.n_heads, cfg.d_ffn, cfg.n_layers).to(dev, dt)
    # a row predicts the token behind it; the prompt's own tokens are given and not scored
    lens = [len(s) - 1 for s in seqs]
    tokens = torch.from_numpy(np.concatenate([s[:-1] for s in seqs])).to(dev)
    labels = torch.from_numpy(np.concatenate([np.where(np.arange(1, len(s)) < P, -1, s[1:]) for s in seqs]).astype(np.int32)).to(dev)
    # both transcripts of an utterance attend to its frames: in training every sequence has its own copy of them
    per = np.split(wl.enc, np.cumsum(wl.enc_lens)[:-1])
    enc = torch.from_numpy(np.concatenate([per[i // 2] for i in range(len(seqs))])).to(dev, dt)
    enc_lens = np.repeat(wl.enc_lens, 2)
    own, cross = model.plans(lens, enc_lens)
    loss_of = training.Preference(lens, cfg.vocab, dt, beta=0.1)
    with torch.no_grad():  # the model that the policy starts from, frozen
        z = model(tokens, enc, own, cross).float()
        ref = torch.log_softmax(z, -1).gather(1, labels.clamp(min=0).long()[:, None])[:, 0].contiguous()
    opt = torch.optim.Adam(model.parameters(), lr=2e-4)
    losses = []
    for step in range(steps):
        opt.zero_grad()
        loss = loss_of.loss(model(tokens, enc, own, cross), labels, ref)
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
        say(f"step {step}: preference loss {losses[-1]:.4f}")
    first = torch.from_numpy(wl.prompt[:, 0].astype(np.int64)).to(dev)
    frames = torch.from_numpy(wl.enc).to(dev, dt)
    written, logits = model.write(first, frames, wl.enc_lens, 12)
    # the same rows once more, all at once
    whole = torch.cat([first[:, None], written[:, :-1]], 1)
    with torch.no_grad():
        packed = model(whole.flatten(), frames, *model.plans([whole.shape[1]] * len(first), wl.enc_lens, training=False)).view_as(logits)
    off = float((packed.float() - logits.float()).abs().max())
    say(f"written one by one: {written[0].tolist()}; largest difference of the logits to all rows at once {off:.2e}")
    return losses, off


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    args = ap.parse_args()
    main(args.steps, args.dtype)
