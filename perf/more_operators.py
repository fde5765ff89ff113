"""Operators on rows of logits, as cases that can be timed and compared: what a program does with what a decoder answers.

Three operators, in the forms that a program next to the decoder uses them in:

  sample   the next token of every sequence of a batch, by temperature, top-k, top-p and min-p, from given random numbers
  top      a teacher's largest logits of every row, with their ids and the mass of all others, to be kept for training
  distill  the divergence of a student's rows from a teacher's largest logits, and its gradient by the student's logits

A case is a dict of plain values:

  op, dtype, rows, vocab   the logits ("bf16" or "fp32")
  sample:
    temperature, top_k, top_p, min_p   of all rows (top_k 0, top_p 1, min_p 0: off), or
    mixed        True: every row has its own, as requests of several users do, greedy ones among them
    banned       share of the ids that the program takes out (logit minus infinity)
  top, distill:
    top          entries of a row's list
    temperature  of the teacher's and the student's distributions
  distill:
    rest         True: what is outside of the list is a class of its own; False: the teacher's list adds up to one
    training     False: forward only, True: forward and the gradient
    unscored     share of the rows with weight 0 (prompts, ends of padded sequences)

`run` has two forms of the same call: elementary torch operations (in 64 bits for sampling, whose borders are looked for
in sums over the whole vocabulary, and for small differences, else in 32) and (own) the framework's kernels.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_SAMPLE = dict(op="sample", dtype="fp32", rows=64, vocab=4096, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mixed=False, banned=0.0)
_TOP = dict(op="top", dtype="bf16", rows=8448, vocab=4096, top=32, temperature=1.0)
_DISTILL = dict(op="distill", dtype="bf16", rows=8448, vocab=4096, top=32, temperature=2.0, rest=True, training=True, unscored=0.1)


def listed():
    return [
        # One live utterance's next token, with the usual three filters: the least a caller asks for.
        dict(_SAMPLE, name="sample_live_b1", rows=1, temperature=0.8, top_k=50, top_p=0.95),
        # A step of the headline configuration's batch as a server has it: every request with its own parameters.
        dict(_SAMPLE, name="sample_mixed_b64", mixed=True, banned=0.01),
        # Nucleus sampling for the 4-layer configuration's batch.
        dict(_SAMPLE, name="sample_nucleus_b256", rows=256, top_p=0.9),
        # The largest batch, unfiltered: transcripts that a policy is tuned on.
        dict(_SAMPLE, name="sample_all_b1024", rows=1024),
        # A wide vocabulary, from a model whose logits are bfloat16.
        dict(_SAMPLE, name="sample_wide_b128", rows=128, vocab=32768, dtype="bf16", temperature=0.7, top_p=0.95, min_p=0.02),
        # The small float32 decoder's rows: 4 sequences of 36 positions.
        dict(_TOP, name="top_tiny", rows=144, vocab=512, dtype="fp32", top=8),
        # A teacher's pass over the headline configuration's batch: 64 sequences of 132 positions.
        dict(_TOP, name="top_b64", temperature=2.0),
        # The same for a wide vocabulary and a long list.
        dict(_TOP, name="top_wide", rows=2048, vocab=32768, top=64),
        # The small decoder scored against a teacher's lists, without a gradient.
        dict(_DISTILL, name="distill_score_tiny", rows=144, vocab=512, dtype="fp32", top=8, temperature=1.0, rest=False, training=False),
        # A training step of the 4-layer decoder on the headline batch.
        dict(_DISTILL, name="distill_train_b64"),
        # The same for long transcripts: 64 sequences of 451 positions.
        dict(_DISTILL, name="distill_train_long", rows=28864, top=16, rest=False),
        # A wide odd vocabulary in float32.
        dict(_DISTILL, name="distill_train_wide", rows=2048, vocab=33000, dtype="fp32", top=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(("sample", "sample", "top", "distill", "distill"))
    dtype = rng.choice(("bf16", "bf16", "fp32"))
    vocab = rng.choice((512, 4096, 4096, 4097, _log(rng, 300, 5000), _log(rng, 5000, 60000)))
    if op == "sample":
        c = dict(_SAMPLE, dtype=rng.choice((dtype, "fp32")), vocab=vocab, rows=_log(rng, 1, min(1024, 4_000_000 // vocab)),
                 temperature=round(rng.uniform(0.3, 1.5), 3), mixed=rng.random() < 0.3, banned=rng.choice((0.0, 0.0, 0.05, 0.5)))
        if rng.random() < 0.4:
            c["top_k"] = _log(rng, 1, min(1000, vocab))
        if rng.random() < 0.5:
            c["top_p"] = round(rng.uniform(0.3, 0.99), 3)
        if rng.random() < 0.3:
            c["min_p"] = round(rng.uniform(0.001, 0.2), 4)
        return c
    top, temperature = min(vocab, rng.choice((1, 8, 16, 32, 64, 128, rng.randint(1, 128)))), rng.choice((1.0, 2.0, 4.0, 0.7))
    if op == "top":
        return dict(_TOP, dtype=dtype, vocab=vocab, rows=_log(rng, 1, min(28000, 60_000_000 // vocab)), top=top, temperature=temperature)
    return dict(_DISTILL, dtype=dtype, vocab=vocab, rows=_log(rng, 1, min(28000, 60_000_000 // vocab)), top=top, temperature=temperature,
                rest=rng.random() < 0.5, training=rng.random() < 0.7, unscored=rng.choice((0.0, 0.1, 0.5)))


# ---------------------------------------------------------------- inputs
def _model_rows(rows, vocab, gen):
    """Logits as a trained model gives them: a bulk, and a few likely continuations, by more or less from row to row."""
    z = 2 * torch.randn((rows, vocab), generator=gen, device="cuda", dtype=torch.float32)
    likely = torch.randint(0, vocab, (rows, 8), generator=gen, device="cuda")
    sure = 0.3 + 0.7 * torch.rand((rows, 1), generator=gen, device="cuda")
    z.scatter_add_(1, likely, sure * (4 + 10 * torch.rand((rows, 8), generator=gen, device="cuda")))
    return z


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    rows, vocab = case["rows"], case["vocab"]
    z = _model_rows(rows, vocab, gen)
    s = {"case": case}
    if own:  # the plan, which a program makes once
        from paper_2503_05931_amd import vocabulary
    if case["op"] == "sample":
        if case["banned"]:
            out = torch.rand((rows, vocab), generator=gen, device="cuda") < case["banned"]
            out[:, 0] = False
            z.masked_fill_(out, -math.inf)
        s["logits"] = z.to(dtype)
        s["uniforms"] = torch.rand(rows, generator=gen, device="cuda")
        if case["mixed"]:
            # greedy; the usual filters; nucleus; likely ones by min-p; unfiltered
            kind = torch.randint(0, 5, (rows,), generator=gen, device="cuda")
            pick = lambda *v, dtype=torch.float32: torch.tensor(v, dtype=dtype, device="cuda")[kind].contiguous()  # noqa: E731
            s["how"] = dict(temperature=pick(0.0, 0.8, 1.0, 1.2, 0.9), top_k=pick(0, 40, 0, 0, 0, dtype=torch.int32),
                            top_p=pick(1.0, 0.95, 0.9, 1.0, 1.0), min_p=pick(0.0, 0.0, 0.0, 0.05, 0.0))
        else:
            s["how"] = {n: case[n] for n in ("temperature", "top_k", "top_p", "min_p")}
        if own:
            s["plan"] = vocabulary.Sampler(vocab, dtype)
        return s
    if case["op"] == "top":
        s["logits"] = z.to(dtype)
        if own:
            s["plan"] = vocabulary.TopLogits(vocab, case["top"], dtype, temperature=case["temperature"])
        return s
    # the student's rows are the teacher's, not quite
    student = 0.9 * z + torch.randn((rows, vocab), generator=gen, device="cuda", dtype=torch.float32)
    s["logits"] = student.to(dtype)
    s["values"], ids = torch.topk(z, case["top"], dim=1)
    s["ids"] = ids.int()
    s["rest"] = torch.logsumexp(z.scatter(1, ids, -math.inf) / case["temperature"], 1) if case["rest"] else None
    scored = torch.rand(rows, generator=gen, device="cuda") >= case["unscored"]
    scored[0] = True
    s["weights"] = scored / scored.sum()
    if own:
        s["plan"] = vocabulary.Distillation(vocab, case["top"], dtype, temperature=case["temperature"])
    return s


# ---------------------------------------------------------------- a pass
def run(s):
    op = s["case"]["op"]
    if op == "sample":
        return _own_sample(s) if own else _plain_sample(s)
    if op == "top":
        return _own_top(s) if own else _plain_top(s)
    return _own_distill(s) if own else _plain_distill(s)


def _own_sample(s):
    tokens, logp = s["plan"].aed_sample(s["logits"], s["uniforms"], **s["how"])
    return {"tokens": tokens, "logp": logp}


def _own_top(s):
    values, ids, rest = s["plan"].aed_top_logits(s["logits"])
    return {"values": values, "ids": ids, "rest": rest}


def _own_distill(s):
    plan, weights = s["plan"], s["weights"]
    loss, row_loss, stats = plan.aed_distill_forward(s["logits"], s["values"], s["ids"], rest=s["rest"], weights=weights)
    if not s["case"]["training"]:
        return {"loss": loss, "row_loss": row_loss}
    d_logits = plan.aed_distill_backward(s["logits"], s["ids"], stats, weights=weights)
    return {"loss": loss, "row_loss": row_loss, "d_logits": d_logits}


def _plain_sample(s):
    z, how = s["logits"].double(), s["how"]
    rows, vocab = z.shape

    def column(name, to):
        v = how[name]
        return v.to(to)[:, None] if torch.is_tensor(v) else torch.tensor(v, device="cuda", dtype=torch.float32).to(to)

    t, k, p, m = column("temperature", torch.float64), column("top_k", torch.int64), column("top_p", torch.float64), column("min_p", torch.float64)
    greedy = ~(t > 0)
    k = torch.where(greedy, 1, torch.where(k > 0, k, vocab))
    ordered, ids = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp((ordered - ordered[:, :1]) / torch.where(greedy, 1.0, t))
    w = torch.where(torch.arange(vocab, device="cuda") < k, w, 0.0)
    through = torch.cumsum(w, 1)
    stays = ((through - w < p * through[:, -1:]) | (p >= 1)) & (w >= m)
    stays[:, 0] = True
    w = torch.zeros_like(w).scatter(1, ids, torch.where(stays, w, 0.0))
    through = torch.cumsum(w, 1)
    total = through[:, -1:]
    tokens = (through <= s["uniforms"].double()[:, None] * total).sum(1)
    logp = torch.log(w.gather(1, tokens[:, None]) / total)[:, 0]
    return {"tokens": tokens.int(), "logp": logp.float()}


def _plain_top(s):
    case = s["case"]
    K, T = case["top"], case["temperature"]
    ordered, ids = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)
    values = ordered[:, :K].contiguous()
    if K == case["vocab"]:
        rest = torch.full_like(values[:, 0], -math.inf)
    else:
        top = ordered[:, K:K + 1]
        rest = top[:, 0] / T + torch.log(torch.exp((ordered[:, K:] - top) / T).sum(1))
    return {"values": values, "ids": ids[:, :K].int(), "rest": rest}


def _plain_distill(s):
    case = s["case"]
    T, ids, weights = case["temperature"], s["ids"].long(), s["weights"]
    # a divergence is a small difference of large logarithms: those of the list and the sums are taken in 64 bits
    z, v = s["logits"].float(), s["values"].double()
    top = z.amax(1, keepdim=True)
    e = torch.exp((z - top) / T)
    listed_e = e.gather(1, ids)
    others = e.scatter(1, ids, 0.0).sum(1, keepdim=True, dtype=torch.float64)
    total = others + listed_e.sum(1, keepdim=True, dtype=torch.float64)
    # the teacher's: log q, with its largest taken off first
    lead = v[:, :1] / T
    log_q = v / T - lead
    norm = torch.exp(log_q).sum(1, keepdim=True)
    if case["rest"]:
        log_rest = s["rest"].double()[:, None] - lead
        norm = norm + torch.exp(log_rest)
    log_q = log_q - torch.log(norm)
    q = torch.exp(log_q)
    log_p = (z.gather(1, ids) - top).double() / T - torch.log(total)
    row = (q * (log_q - log_p)).sum(1)
    off = 1.0
    if case["rest"]:
        log_rest = log_rest - torch.log(norm)
        q_rest = torch.exp(log_rest)
        row = row + (q_rest * (log_rest - torch.log(others / total)))[:, 0]
        off = 1 - q_rest * total / others
    row = torch.where(weights != 0, T * T * row, 0.0)
    loss = (weights * row).sum()
    if not case["training"]:
        return {"loss": loss.float(), "row_loss": row.float()}
    slope = (T * weights)[:, None]
    d = (slope * off / total).float() * e
    d = d.scatter(1, ids, (slope * (listed_e / total - q)).float())
    return {"loss": loss.float(), "row_loss": row.float(), "d_logits": d.to(s["logits"].dtype)}


# ---------------------------------------------------------------- in 64 bits, from the definitions
def exact(case, seed):
    s = prepare(case, seed)
    return {"sample": _exact_sample, "top": _exact_top, "distill": _exact_distill}[case["op"]](s)


def _exact_sample(s):
    case = s["case"]
    logits, uniforms = s["logits"].float().cpu().numpy().astype(np.float64), s["uniforms"].cpu().numpy().astype(np.float64)
    how = {n: np.broadcast_to(np.asarray(v.cpu() if torch.is_tensor(v) else np.float32(v)), (case["rows"],)).astype(np.float64) for n, v in s["how"].items()}
    tokens, logps = [], []
    for r, z in enumerate(logits):
        t, k, p, m = (how[n][r] for n in ("temperature", "top_k", "top_p", "min_p"))
        first = int(np.argmax(z))
        if t <= 0:
            tokens.append(first)
            logps.append(0.0)
            continue
        left = np.flatnonzero(np.isfinite(z))
        left = left[np.argsort(-z[left], kind="stable")]
        if k > 0:
            left = left[:int(k)]
        w = np.exp((z[left] - z[first]) / t)
        if p < 1:
            before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
            count = max(1, int(np.count_nonzero(before < p * w.sum())))
            left, w = left[:count], w[:count]
        use = w >= m
        left, w = left[use], w[use]
        by_id = np.argsort(left)
        left, w = left[by_id], w[by_id]
        sums = np.cumsum(w)
        at = int(np.searchsorted(sums, uniforms[r] * sums[-1], side="right"))
        tokens.append(int(left[at]))
        logps.append(math.log(w[at] / sums[-1]))
    return {"tokens": torch.tensor(tokens, dtype=torch.int32), "logp": torch.tensor(logps, dtype=torch.float64)}


def _exact_top(s):
    case = s["case"]
    K, T = case["top"], case["temperature"]
    values, ids, rests = [], [], []
    for z in s["logits"].split(max(1, (1 << 24) // case["vocab"])):
        z = z.double()
        z_host = z.cpu().numpy()
        # the K-th largest value: all above it, and of its equals those with the lowest ids
        border = -np.partition(-z_host, K - 1, axis=1)[:, K - 1:K]
        equal = z_host == border
        room = K - (z_host > border).sum(1, keepdims=True)
        chosen = (z_host > border) | (equal & (np.cumsum(equal, 1) <= room))
        at = np.nonzero(chosen)[1].reshape(-1, K)  # ids rise
        value = np.take_along_axis(z_host, at, 1)
        order = np.argsort(-value, axis=1, kind="stable")
        values.append(np.take_along_axis(value, order, 1))
        ids.append(np.take_along_axis(at, order, 1))
        rests.append(torch.logsumexp((z / T).masked_fill(torch.from_numpy(chosen).cuda(), -math.inf), 1))
    return {"values": torch.from_numpy(np.concatenate(values)), "ids": torch.from_numpy(np.concatenate(ids)).int(), "rest": torch.cat(rests)}


def _exact_distill(s):
    case = s["case"]
    T, grads, rows = case["temperature"], [], []
    step = max(1, (1 << 24) // case["vocab"])
    for a in range(0, case["rows"], step):
        part = slice(a, a + step)
        z = s["logits"][part].double().requires_grad_(case["training"])
        ids, weights = s["ids"][part].long(), s["weights"][part].double()
        teacher = s["values"][part].double() / T
        student = torch.log_softmax(z / T, 1)
        theirs = student.gather(1, ids)
        if case["rest"]:
            teacher = torch.cat((teacher, s["rest"][part].double()[:, None]), 1)
            theirs = torch.cat((theirs, torch.logsumexp(student.scatter(1, ids, -math.inf), 1, keepdim=True)), 1)
        teacher = torch.log_softmax(teacher, 1)
        row = T ** 2 * torch.nn.functional.kl_div(theirs, teacher, reduction="none", log_target=True).sum(1)
        if case["training"]:
            (row * weights).sum().backward()
            grads.append(z.grad)
        rows.append(torch.where(weights != 0, row.detach(), 0.0))
    rows = torch.cat(rows)
    got = {"loss": (rows * s["weights"].double()).sum(), "row_loss": rows}
    return got | ({"d_logits": torch.cat(grads)} if case["training"] else {})


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    """Inputs once, outputs once; of an element: a difference, a scale, an exponential and a sum, and as many for the gradient."""
    e = 2 if case["dtype"] == "bf16" else 4
    rows, elements = case["rows"], case["rows"] * case["vocab"]
    if case["op"] == "sample":
        return {"bytes": float(elements * e + rows * (12 + (16 if case["mixed"] else 0))), "flops": 4.0 * elements}
    if case["op"] == "top":
        return {"bytes": float(elements * e + rows * (8 * case["top"] + 4)), "flops": 4.0 * elements}
    scored = 1 - case["unscored"]  # of rows that are not scored only the gradient is written
    read = scored * rows * (case["vocab"] * e + 8 * case["top"] + 4) + 8 * rows
    return {"bytes": float(read + (elements * e if case["training"] else 0)), "flops": (8.0 if case["training"] else 4.0) * elements * scored}
