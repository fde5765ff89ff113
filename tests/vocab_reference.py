"""Plain float64 forms of the operators on rows of logits (not collected by pytest): one row at a time, from the definitions in
include/aed_vocab.h."""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np
import torch


def order(z):
    """Ids in the row's order; without those of minus infinity and NaN."""
    z = np.asarray(z, np.float64)
    return sorted((i for i in range(len(z)) if z[i] > -math.inf), key=lambda i: (-z[i], i))


def units(x):
    """A float64 as a whole multiple of 2^-1074: sums are exact."""
    m, e = math.frexp(x)
    return int(m * 2.0 ** 53) << (e - 53 + 1074) if e - 53 + 1074 >= 0 else int(m * 2.0 ** 53) >> -(e - 53 + 1074)


def left_of(z, t=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(ids in the row's order, weights in units) of what the filters leave."""
    z = np.asarray(z, np.float64)
    ids = order(z)
    if not ids:
        return [], []
    t, top_p, min_p = float(t), float(top_p), float(min_p)
    if not t > 0:
        return ids[:1], [units(1.0)]
    if 0 < top_k < len(z):
        ids = ids[:top_k]
    top = z[ids[0]]
    w = [1.0 if z[i] == top else 0.0 if top == math.inf else math.exp((z[i] - top) / t) for i in ids]
    least = min(min_p, 1.0) if min_p > 0 else 0.0
    keep = [x >= least for x in w]
    w = [units(x) for x in w]
    if top_p < 1:
        border, front, n = Fraction(max(top_p, 0.0)) * sum(w), 0, 0
        for x in w:
            if n > 0 and not front < border:
                break
            front, n = front + x, n + 1
        ids, w = ids[:n], w[:n]
    return [i for i, k in zip(ids, keep) if k], [x for x, k in zip(w, keep) if k]


def sample(z, u, **how):
    """(token, log-probability)"""
    ids, w = left_of(z, **how)
    if not ids:
        return -1, -math.inf
    total = sum(w)
    border = Fraction(min(max(float(u), 0.0), 1.0) if u == u else 0.0) * total
    through, last = 0, None
    for i, x in sorted(zip(ids, w)):
        through += x
        if x > 0:
            last = i, math.log(x / total)
            if through > border:
                return last
    return last


def top_logits(z, top, t):
    """(values, ids, rest)"""
    z = np.asarray(z, np.float64)
    ids = order(z)
    others = z[ids[top:]]
    rest = -math.inf
    if len(others):
        m = others.max()
        rest = math.inf if m == math.inf else m / t + math.log(math.fsum(np.exp((others - m) / t)))
    ids = ids[:top]
    fill = top - len(ids)
    return list(z[ids]) + [-math.inf] * fill, ids + [-1] * fill, rest


def distill_row(z, values, ids, rest, t):
    """L of a row in float64; differentiable by z (a float64 tensor)."""
    vocab = z.shape[0]
    entries = [(int(i), float(v)) for i, v in zip(ids, values) if 0 <= int(i) < vocab and float(v) != -math.inf]
    logs = [v / t for _, v in entries] + ([] if rest is None else [float(rest)])
    lead = max(logs, default=-math.inf)
    if lead == -math.inf:
        return 0.0 * torch.nan_to_num(z, 0.0, 0.0, 0.0).sum()
    log_n = lead + math.log(math.fsum(math.exp(x - lead) for x in logs))
    top = z.max()
    if top == -math.inf:
        log_p = torch.full_like(z, -math.inf)
    else:
        z = (z - top.detach()) / t  # first of all: logits of 1e20 have no place for a sum's log, not in 64 bits either
        log_p = z - torch.logsumexp(z, 0)
    total = torch.zeros((), dtype=torch.float64)
    for i, v in entries:
        log_q = v / t - log_n
        if math.exp(log_q) > 0:
            total = total + math.exp(log_q) * (log_q - log_p[i])
    if rest is not None and math.exp(float(rest) - log_n) > 0:
        out = torch.ones(vocab, dtype=torch.bool)
        out[[i for i, _ in entries]] = False
        others = torch.logsumexp(log_p[out], 0) if bool(out.any()) else torch.tensor(-math.inf, dtype=torch.float64)
        total = total + math.exp(float(rest) - log_n) * (float(rest) - log_n - others)
    return t * t * total


def distill(z, values, ids, rest, weights, t):
    """(loss, row losses) in float64; differentiable by z."""
    n = z.shape[0]
    rows = []
    for r in range(n):
        w = 1 / n if weights is None else float(weights[r])
        rows.append(torch.zeros((), dtype=torch.float64) if w == 0 else distill_row(z[r], values[r], ids[r], None if rest is None else rest[r], t))
    rows = torch.stack(rows)
    if weights is None:
        return rows.mean(), rows
    use = weights.double() != 0
    return (rows[use] * weights.double()[use]).sum(), rows


def distill_gradient(z, values, ids, rest, weights, t):
    """The formula of the header, in float64."""
    n, vocab = z.shape
    d = torch.zeros((n, vocab), dtype=torch.float64)
    for r in range(n):
        w = 1 / n if weights is None else float(weights[r])
        if w == 0:
            continue
        entries = [(int(i), float(v)) for i, v in zip(ids[r], values[r]) if 0 <= int(i) < vocab and float(v) != -math.inf]
        logs = [v / t for _, v in entries] + ([] if rest is None else [float(rest[r])])
        lead = max(logs, default=-math.inf)
        if lead == -math.inf:
            continue
        log_n = lead + math.log(math.fsum(math.exp(x - lead) for x in logs))
        x = z[r].double()
        x = (x - (0 if x.max() == -math.inf else x.max())) / t
        log_p = torch.full_like(x, -math.inf) if x.max() == -math.inf else x - torch.logsumexp(x, 0)
        out = torch.ones(vocab, dtype=torch.bool)
        out[[i for i, _ in entries]] = False
        d[r] = torch.exp(log_p)
        if rest is not None and float(rest[r]) > -math.inf and bool(out.any()) and log_p[out].max() > -math.inf:
            d[r][out] -= math.exp(float(rest[r]) - log_n) * torch.softmax(x[out], 0)  # p_i / p_R
        for i, v in entries:
            d[r][i] -= math.exp(v / t - log_n)
        d[r] *= w * t
    return d
