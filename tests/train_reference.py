"""Plain float64 forms of the training operators (not collected by pytest): one sequence, one head and one row at a time,
from the definitions in include/aed_train.h."""
from __future__ import annotations

import math

import torch


def bucket(n, buckets, max_distance, bidirectional):
    """Bucket of the distance n = place of the query - place of the key, in whole numbers."""
    side = buckets // 2 if bidirectional else buckets
    first = side if bidirectional and n < 0 else 0
    n = abs(n) if bidirectional else max(n, 0)
    half = side // 2
    if n < half:
        return first + n
    b = half
    while b + 1 < side and n ** (side - half) * half ** (b + 1 - half) >= half ** (side - half) * max_distance ** (b + 1 - half):
        b += 1
    return first + b


def attention(q, k, v, q_lens, k_lens, scale=None, causal=False, bias=None, max_distance=0, bidirectional=False, key_mask=None, k_starts=None):
    """(out, lse) in float64; differentiable by q, k, v and bias."""
    H, G, D = q.shape[1], k.shape[1], q.shape[2]
    scale = 1 / math.sqrt(D) if scale is None else scale
    row, packed, outs, lses = 0, 0, [], []
    for b, (nq, nk) in enumerate(zip(q_lens, k_lens)):
        at = packed if k_starts is None else int(k_starts[b])
        far = [[i + nk - nq - j for j in range(nk)] for i in range(nq)]
        seen = torch.tensor([[(not causal or n >= 0) for n in line] for line in far], dtype=torch.bool).reshape(nq, nk)
        if key_mask is not None:
            seen = seen & (key_mask[at:at + nk] != 0)[None, :]
        if bias is not None:
            place = {n: bucket(n, bias.shape[0], max_distance, bidirectional) for line in far for n in line}
            place = torch.tensor([[place[n] for n in line] for line in far], dtype=torch.long).reshape(nq, nk)
        rows, stats = [], []
        for h in range(H):
            g = h // (H // G)
            # what is not seen does not count, whatever it holds
            some = seen.any(0)
            kk = torch.where(some[:, None], k[at:at + nk, g], torch.zeros((), dtype=torch.float64))
            vv = torch.where(some[:, None], v[at:at + nk, g], torch.zeros((), dtype=torch.float64))
            s = q[row:row + nq, h] @ kk.T * scale
            if bias is not None:
                s = s + bias[place, h]
            s = torch.where(seen, s, torch.full((), -1e30, dtype=torch.float64))
            top = s.max(1, keepdim=True).values.detach() if nk else torch.zeros((nq, 1), dtype=torch.float64)
            e = torch.exp(s - top) * seen
            total = e.sum(1, keepdim=True)
            empty = total == 0
            rows.append((e / torch.where(empty, torch.ones_like(total), total)) @ vv)
            stats.append(torch.where(empty, torch.full_like(total, -math.inf), top + torch.log(total))[:, 0])
        outs.append(torch.stack(rows, 1))
        lses.append(torch.stack(stats, 1))
        row += nq
        packed += nk
    return torch.cat(outs), torch.cat(lses)


def attention_gradients(q, k, v, d_out, q_lens, k_lens, bias=None, **kw):
    """(out, lse, dq, dk, dv, d_bias or None)"""
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)] + ([bias.clone().requires_grad_(True)] if bias is not None else [])
    out, lse = attention(leaves[0], leaves[1], leaves[2], q_lens, k_lens, bias=leaves[3] if bias is not None else None, **kw)
    grads = torch.autograd.grad((out * d_out).sum(), leaves, allow_unused=True)
    grads = [torch.zeros_like(t) if g is None else g for t, g in zip(leaves, grads)]
    return out.detach(), lse.detach(), grads[0], grads[1], grads[2], grads[3] if bias is not None else None


def attention_bounds(q, k, v, d_out, q_lens, k_lens, u, scale=None, causal=False, bias=None, max_distance=0, bidirectional=False, key_mask=None):
    """How far each element of (out, dq, dk, dv, d_bias) may be off when weights and results are rounded to u of themselves:
    the formulas with magnitudes in the place of numbers.  out: the weights' rounding and its own.  delta of dq and d_bias is
    that of the rounded output; dk's and dv's is exact."""
    H, G, D = q.shape[1], k.shape[1], q.shape[2]
    scale = 1 / math.sqrt(D) if scale is None else scale
    e_out, e_dq, e_dk, e_dv = (torch.zeros_like(t) for t in (q, q, k, v))
    e_bias = None if bias is None else torch.zeros_like(bias)
    row = at = 0
    for nq, nk in zip(q_lens, k_lens):
        qs, ks = slice(row, row + nq), slice(at, at + nk)
        far = torch.arange(nq)[:, None] + nk - nq - torch.arange(nk)[None, :]
        seen = torch.ones((nq, nk), dtype=torch.bool) if not causal else far >= 0
        if key_mask is not None:
            seen = seen & (key_mask[ks] != 0)[None, :]
        if bias is not None:
            place = far.clone().apply_(lambda n: bucket(int(n), bias.shape[0], max_distance, bidirectional))
        for h in range(H):
            g = h // (H // G)
            s = q[qs, h] @ k[ks, g].T * scale + (bias[place, h] if bias is not None else 0)
            p = torch.nan_to_num(torch.softmax(torch.where(seen, s, torch.full((), -math.inf, dtype=torch.float64)), 1)) if nk else s
            out, do = p @ v[ks, g], d_out[qs, h]
            err = u * (out.abs() + p @ v[ks, g].abs())
            ds = p * (do @ v[ks, g].T - (do * out).sum(1, keepdim=True))
            off_ds = u * ds.abs()
            off_row = off_ds + p * (do.abs() * err).sum(1, keepdim=True)
            e_out[qs, h] = err
            e_dq[qs, h] = scale * off_row @ k[ks, g].abs()
            e_dk[ks, g] += scale * off_ds.T @ q[qs, h].abs()
            e_dv[ks, g] += u * p.T @ do.abs()
            if bias is not None:
                e_bias[:, h].index_add_(0, place.reshape(-1), (p * (do.abs() * err).sum(1, keepdim=True)).reshape(-1))
        row += nq
        at += nk
    return e_out, e_dq, e_dk, e_dv, e_bias


def preference(logits, labels, ref, seq_lens, beta, smoothing):
    """(loss, ratio) in float64; differentiable by the logits."""
    vocab = logits.shape[1]
    row, ratio = 0, []
    for n in seq_lens:
        total = torch.zeros((), dtype=torch.float64)
        for t in range(row, row + n):
            y = int(labels[t])
            if 0 <= y < vocab:
                total = total + logits[t, y] - torch.logsumexp(logits[t], 0) - ref[t]
        ratio.append(total)
        row += n
    ratio = torch.stack(ratio)
    x = beta * (ratio[0::2] - ratio[1::2])

    def cost(y):  # -log sigmoid
        return torch.log1p(torch.exp(-y.abs())) + (-y).clamp(min=0)

    return ((1 - smoothing) * cost(x) + smoothing * cost(-x)).mean(), ratio


def off(x, y):
    """(2-norm of the difference over that of y, largest difference over max(|y|, rms of y)); finite places have to agree."""
    x, y = x.double().cpu(), y.double().cpu()
    assert x.shape == y.shape
    fine = torch.isfinite(y)
    assert torch.equal(fine, torch.isfinite(x)) and torch.equal(x[~fine], y[~fine])
    x, y = x[fine], y[fine]
    if y.numel() == 0 or not bool(y.any()):
        return float(x.abs().max()) if x.numel() else 0.0, 0.0
    rms = float(y.norm()) / math.sqrt(y.numel())
    return float((x - y).norm() / y.norm()), float(((x - y).abs() / y.abs().clamp(min=rms)).max())
