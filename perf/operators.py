"""Operators on rows of scores [B, T, W]: the cases that are measured, and the
operators' plain forms.

  process  logits -> log-probabilities, with penalties for tokens that were
           emitted before, biases and grammar masks
  top      the k largest logits of a row and the log-sum of the others
  distill  the divergence from a teacher's top logits, and its gradient

``own`` False: elementary torch operations.  ``own`` True: the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

LARGEST = float(torch.finfo(torch.float32).max)
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}


# --------------------------------------------------------------------- cases

def listed():
    return [
        # one stream's next frame, a handful of tokens emitted so far: latency
        dict(name="process one frame", op="process", B=1, T=1, W=1025, type="fp32", H=24, ragged=False,
             bias="none", mask="none", normalize=True),
        # a decoding step of many requests: long histories, a grammar and penalties of each request's own
        dict(name="process step of 64 requests", op="process", B=64, T=1, W=131072, type="bf16", H=2048, ragged=False,
             bias="none", mask="row", normalize=True),
        # a step of few requests over an odd vocabulary, scores for a sampler (not normalised), a bias of each request
        dict(name="process step, raw scores", op="process", B=12, T=1, W=32003, type="fp16", H=700, ragged=False,
             bias="row", mask="row", normalize=False),
        # a batch of utterances for the decoder: 1024 tokens and blank, one bias for all, labels barred per utterance
        dict(name="process utterances", op="process", B=64, T=400, W=1025, type="fp32", H=40, ragged=True,
             bias="shared", mask="row", normalize=True),
        # a grammar that moves from frame to frame, the decoder's largest vocabulary
        dict(name="process frames, moving mask", op="process", B=16, T=250, W=4097, type="bf16", H=0, ragged=True,
             bias="none", mask="frame", normalize=True),
        # a short utterance over a letter vocabulary
        dict(name="top of a short utterance", op="top", B=1, T=50, W=33, type="fp32", k=4, ragged=False),
        # a teacher's frames, kept for training
        dict(name="top of utterances", op="top", B=64, T=400, W=1025, type="bf16", k=16, ragged=True),
        # a teacher's rows over a large odd vocabulary
        dict(name="top of a large vocabulary", op="top", B=4, T=512, W=65537, type="bf16", k=64, ragged=False),
        # a training step on utterances: loss and gradient at once
        dict(name="distill utterances", op="distill", B=64, T=400, W=1025, type="bf16", k=16, ragged=True,
             tail=True, temperature=1.0, loss=True, grad=True),
        # a validation pass: loss alone
        dict(name="distill loss", op="distill", B=8, T=300, W=4097, type="fp32", k=32, ragged=True,
             tail=True, temperature=1.0, loss=True, grad=False),
        # the backward pass of a small model's last utterances, the teacher's list renormalised
        dict(name="distill gradient", op="distill", B=8, T=90, W=513, type="fp16", k=8, ragged=True,
             tail=False, temperature=2.0, loss=False, grad=True),
        # a training step over a large vocabulary: the largest work
        dict(name="distill a large vocabulary", op="distill", B=2, T=1024, W=131072, type="bf16", k=64, ragged=False,
             tail=True, temperature=1.0, loss=True, grad=True),
    ]


def _spread(rng, low, high):
    """A whole number between low and high, spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["process", "process", "top", "distill", "distill"])
    kind = rng.choice(["fp32", "bf16", "fp16"])
    W = _spread(rng, 5, 140000)
    most = (1 << 27) // W                     # half the largest listed case's labels
    if op == "process" and rng.random() < 0.5:
        B, T = _spread(rng, 1, max(1, min(256, most // 2))), 1
    else:
        B = _spread(rng, 1, max(1, min(64, most // 2)))
        T = _spread(rng, 1, max(1, min(1024, most // (2 * B))))
    case = dict(op=op, B=B, T=T, W=W, type=kind, ragged=T > 1 and rng.random() < 0.7)
    if op == "process":
        case.update(H=rng.choice([0, _spread(rng, 1, 8192)]), bias=rng.choice(["none", "shared", "row"]),
                    mask=rng.choice(["none", "row", "frame"]), normalize=rng.random() < 0.8)
    else:
        case.update(k=_spread(rng, 1, min(W, 128)))
    if op == "distill":
        loss = rng.random() < 0.7
        case.update(tail=rng.random() < 0.7, temperature=rng.choice([1.0, 0.7, 2.0, 4.0]), loss=loss,
                    grad=not loss or rng.random() < 0.7)
    return case


# -------------------------------------------------------------------- inputs

def _logits(case, g, dev):
    """Scores N(0, 2^2); as in a model's frames, most rows have a label that stands out."""
    B, T, W = case["B"], case["T"], case["W"]
    x = torch.randn((B, T, W), generator=g, device=dev, dtype=torch.float32).mul_(2.0)
    peak = torch.randint(0, W, (B, T, 1), generator=g, device=dev)
    if T > 1:                                  # frames: the last label (blank) leads in 70 of 100
        blank = torch.rand((B, T, 1), generator=g, device=dev) < 0.7
        peak = torch.where(blank, torch.full_like(peak, W - 1), peak)
    high = torch.rand((B, T, 1), generator=g, device=dev).mul_(6.0).add_(3.0)
    x.scatter_add_(2, peak, high)
    return x.to(TYPES[case["type"]])


def _lengths(case, g, dev):
    B, T = case["B"], case["T"]
    if not case["ragged"]:
        return None
    return torch.randint((T + 1) // 2, T + 1, (B,), generator=g, device=dev, dtype=torch.int32)


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    B, T, W, op = case["B"], case["T"], case["W"], case["op"]
    s = dict(case=case, op=op)
    s["logits"] = _logits(case, g, dev)
    s["lengths"] = _lengths(case, g, dev)
    if op == "process":
        H = case["H"]
        s["history"] = s["history_lengths"] = s["penalties"] = s["bias"] = s["mask"] = None
        if H:
            # tokens repeat: small ids are frequent ones; -1 pads
            u = torch.rand((B, H), generator=g, device=dev)
            s["history"] = (u * u * u * W).to(torch.int32).clamp_(0, W - 1)
            hl = torch.randint(H // 2, H + 1, (B,), generator=g, device=dev, dtype=torch.int32)
            behind = torch.arange(H, device=dev)[None] >= hl[:, None]
            s["history"].masked_fill_(behind, -1)
            s["history_lengths"] = hl
            p = torch.rand((B, 3), generator=g, device=dev)
            p[:, 0].mul_(0.4).add_(1.0)        # repetition 1.0 .. 1.4
            s["penalties"] = p.contiguous()    # presence and frequency 0 .. 1
        if case["bias"] != "none":
            s["bias"] = torch.randn((W,) if case["bias"] == "shared" else (B, W), generator=g, device=dev)
        if case["mask"] != "none":
            words = (W + 31) // 32
            shape = (B, words) if case["mask"] == "row" else (B, T, words)
            r = [torch.randint(-2**31, 2**31, shape, generator=g, device=dev, dtype=torch.int64) for _ in range(2)]
            s["mask"] = (r[0] | r[1]).to(torch.int32)          # three labels in four are allowed
        s["out"] = torch.zeros((B, T, W), device=dev)
    if op == "distill":
        k = case["k"]
        vs, ids, rest = [], [], []
        step = max(1, (1 << 26) // W)
        rows = s["logits"].view(B * T, W)
        for at in range(0, B * T, step):
            x = rows[at:at + step].float()
            x = x.mul(1.2).add_(torch.randn(x.shape, generator=g, device=dev))
            v, i = torch.topk(x, k, dim=1)
            x.scatter_(1, i, -math.inf)
            vs.append(v)
            ids.append(i.to(torch.int32))
            rest.append(torch.logsumexp(x / case["temperature"], 1))
        s["values"] = torch.cat(vs).view(B, T, k)
        s["ids"] = torch.cat(ids).view(B, T, k)
        s["tail"] = torch.cat(rest).view(B, T) if case["tail"] else None
        s["weights"] = torch.rand((B, T), generator=g, device=dev).add_(0.5)
    return s


# --------------------------------------------------------------- plain forms

def _valid(lengths, B, T, dev):
    """[B, T]: the frames that an utterance has."""
    t = torch.arange(T, device=dev)[None]
    if lengths is None:
        return (t >= 0).expand(B, T)
    return t < lengths[:, None].clamp(0, T)


def _clean(x):
    """NaN counts as -inf, +inf as the largest number."""
    return torch.where(torch.isnan(x), -math.inf, x).clamp(max=LARGEST)


def _log_sum(x):
    """log sum exp over the last axis; -inf where it holds nothing."""
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    return m + torch.log(torch.exp(x - m).sum(-1, keepdim=True))


def _process(logits, lengths, history, history_lengths, penalties, bias, mask, normalize, kind):
    B, T, W = logits.shape
    dev = logits.device
    x = _clean(logits.to(kind))
    if history is not None:
        H = history.shape[1]
        real = (torch.arange(H, device=dev)[None] < history_lengths[:, None]) & (history >= 0) & (history < W)
        at = torch.where(real, history, 0).long()
        n = torch.zeros((B, W), device=dev, dtype=kind).scatter_add_(1, at, real.to(kind))[:, None]
        r, p, f = (penalties[:, i].to(kind)[:, None, None] for i in range(3))
        seen = torch.where(x > 0, x / r, x * r) - f * n - p
        x = torch.where(n > 0, seen, x)
    if bias is not None:
        x = x + (bias if bias.dim() == 1 else bias[:, None])
    x = _clean(x)
    if mask is not None:
        bits = (mask[..., :, None] >> torch.arange(32, device=dev, dtype=torch.int32)) & 1
        bits = bits.flatten(-2)[..., :W] != 0
        x = torch.where(bits if mask.dim() == 3 else bits[:, None], x, -math.inf)
    if normalize:
        total = _log_sum(x)
        x = x - torch.where(total == -math.inf, 0.0, total)
    return x


def _top(logits, lengths, k, temperature, kind):
    B, T, W = logits.shape
    x = _clean(logits.to(kind))
    v, i = torch.sort(x, dim=-1, descending=True, stable=True)     # equal values: the lowest index first
    values, ids = v[..., :k], i[..., :k].to(torch.int32)
    tail = _log_sum(v[..., k:] / temperature).squeeze(-1) if k < W else torch.full_like(v[..., 0], -math.inf)
    there = _valid(lengths, B, T, logits.device)
    return (torch.where(there[..., None], values, -math.inf), torch.where(there[..., None], ids, -1),
            torch.where(there, tail, -math.inf))


def _distill(student, values, ids, tail, lengths, temperature, weights, loss, grad, kind):
    B, T, W = student.shape
    s = 1.0 / temperature
    x = student.to(kind) * s
    real = (ids >= 0) & (ids < W) & (values > -math.inf)
    u = torch.where(real, values.to(kind) * s, -math.inf)
    rest = torch.full((B, T, 1), -math.inf, device=x.device, dtype=kind) if tail is None else tail[..., None].to(kind)
    both = torch.cat([u, rest], -1)
    total = _log_sum(both)
    some = total > -math.inf
    log_p = both - torch.where(some, total, 0.0)
    p = torch.exp(log_p)
    at = torch.where(real, ids, 0).long()
    P = torch.zeros_like(x).scatter_add_(2, at, torch.where(real, p[..., :-1], 0.0))
    is_listed = torch.zeros_like(x, dtype=torch.int32).scatter_add_(2, at, real.to(torch.int32)) > 0
    own_total = _log_sum(x)
    use = _valid(lengths, B, T, x.device)[..., None] & some & (own_total > -math.inf)
    log_q = x - own_total
    rest_total = _log_sum(torch.where(is_listed, -math.inf, x))
    out = []
    if loss:
        terms = torch.where(P > 0, P * (torch.log(torch.where(P > 0, P, 1.0)) - log_q), 0.0).sum(-1, keepdim=True)
        pr, log_qr = p[..., -1:], rest_total - own_total
        terms = terms + torch.where(pr > 0, pr * (log_p[..., -1:] - log_qr), 0.0)
        out.append(torch.where(use, terms, 0.0).squeeze(-1))
    if grad:
        q = torch.exp(log_q)
        in_rest = torch.exp(x - torch.where(rest_total == -math.inf, 0.0, rest_total))
        g = torch.where(is_listed, q - P, q - p[..., -1:] * in_rest)
        g = torch.where(use, g * (weights[..., None] * s), 0.0)
        out.append(g)
    return out


# ----------------------------------------------------------------------- run

def run(state):
    s, c = state, state["case"]
    if own:
        import paper_2508_07315_amd as ctcbeam
        if s["op"] == "process":
            return ctcbeam.process_logits(s["logits"], s["lengths"], history=s["history"],
                                          history_lengths=s["history_lengths"], penalties=s["penalties"],
                                          bias=s["bias"], mask=s["mask"], normalize=c["normalize"], out=s["out"])
        if s["op"] == "top":
            return ctcbeam.top_logits(s["logits"], c["k"], s["lengths"])
        loss, grad = ctcbeam.distill(s["logits"], s["values"], s["ids"], s["tail"], s["lengths"],
                                     temperature=c["temperature"], weights=s["weights"],
                                     want_loss=c["loss"], want_grad=c["grad"])
        return [t for t in (loss, grad) if t is not None]
    if s["op"] == "process":
        x = _process(s["logits"], s["lengths"], s["history"], s["history_lengths"], s["penalties"], s["bias"],
                     s["mask"], c["normalize"], torch.float32)
        there = _valid(s["lengths"], c["B"], c["T"], x.device)[..., None]
        return s["out"].copy_(torch.where(there, x, s["out"]))
    if s["op"] == "top":
        return _top(s["logits"], s["lengths"], c["k"], 1.0, torch.float32)
    out = _distill(s["logits"], s["values"], s["ids"], s["tail"], s["lengths"], c["temperature"], s["weights"],
                   c["loss"], c["grad"], torch.float32)
    if c["grad"]:
        out[-1] = out[-1].to(s["logits"].dtype)
    return out


def work(case):
    B, T, W, e = case["B"], case["T"], case["W"], SIZE[case["type"]]
    there = (0.5 * ((T + 1) // 2 + T) / T) if case["ragged"] else 1.0     # the mean share of frames that are there
    rows = B * T * there
    if case["op"] == "process":
        words = 4 * ((W + 31) // 32)
        n = rows * W * (e + 4) + 3 * B * case["H"]
        n += {"none": 0, "shared": 4 * W, "row": 4 * B * W}[case["bias"]]
        n += {"none": 0, "row": B * words, "frame": rows * words}[case["mask"]]
        return {"bytes": n, "flops": 8 * rows * W}
    k = case["k"]
    if case["op"] == "top":
        return {"bytes": rows * W * e + B * T * (8 * k + 4), "flops": 4 * rows * W}
    n = rows * (W * e + 8 * k + 8)
    n += B * T * W * e if case["grad"] else 0
    return {"bytes": n, "flops": (6 + 3 * case["grad"]) * rows * W}


# --------------------------------------------------------------- in 64 bits

def exact(case, seed):
    """The operators from their definitions, in 64 bits, a block of rows at a time."""
    s = prepare(case, seed)
    B, T, W = case["B"], case["T"], case["W"]
    D = torch.float64
    x_all = s["logits"].reshape(B * T, W)
    dev = x_all.device
    length = torch.full((B,), T, device=dev) if s["lengths"] is None else s["lengths"]
    utt = torch.arange(B * T, device=dev) // T
    there_all = (torch.arange(B * T, device=dev) % T) < length[utt]
    step = max(1, (1 << 25) // W)
    parts = []
    for at in range(0, B * T, step):
        sl = slice(at, min(at + step, B * T))
        x = x_all[sl].to(D)
        b, there = utt[sl], there_all[sl]
        if case["op"] == "process":
            if s["history"] is not None:
                n = torch.zeros((B, W + 1), device=dev, dtype=D)
                h = torch.where(s["history"] < 0, W, s["history"]).long()
                n.scatter_add_(1, h, torch.ones_like(h, dtype=D))
                n = n[:, :W][b]
                pen = s["penalties"].to(D)[b]
                seen = torch.maximum(x, torch.zeros_like(x)) / pen[:, :1] + torch.minimum(x, torch.zeros_like(x)) * pen[:, :1]
                x = torch.where(n > 0, seen - pen[:, 1:2] - pen[:, 2:] * n, x)
            if s["bias"] is not None:
                x = x + (s["bias"].to(D).expand(B, W))[b]
            if s["mask"] is not None:
                w = s["mask"].reshape(-1, s["mask"].shape[-1])
                w = w[b] if s["mask"].dim() == 2 else w[sl]
                c = torch.arange(W, device=dev)
                ok = ((w[:, c // 32].long() >> (c % 32)) & 1).bool()
                x = x.masked_fill(~ok, -math.inf)
            if case["normalize"]:
                x = torch.nan_to_num(torch.log_softmax(x, 1), nan=-math.inf, neginf=-math.inf)
            parts.append((x.masked_fill(~there[:, None], 0.0).to(torch.float32) if W * B * T > (1 << 27)
                          else x.masked_fill(~there[:, None], 0.0),))
        elif case["op"] == "top":
            k = case["k"]
            v, i = torch.topk(x, k, dim=1)
            rest = torch.logsumexp(x.scatter(1, i, -math.inf), 1)
            parts.append((v.masked_fill(~there[:, None], -math.inf), rest.masked_fill(~there, -math.inf)))
        else:
            tau, k = case["temperature"], case["k"]
            ids = s["ids"].reshape(-1, k)[sl].long()
            v = s["values"].reshape(-1, k)[sl].to(D) / tau
            rest = s["tail"].reshape(-1, 1)[sl].to(D) if s["tail"] is not None else torch.full((len(v), 1), -math.inf, device=dev, dtype=D)
            log_p = torch.log_softmax(torch.cat([v, rest], 1), 1)       # the ids of a row differ
            log_q = torch.log_softmax(x / tau, 1)
            log_qr = torch.logsumexp(log_q.scatter(1, ids, -math.inf), 1, keepdim=True)
            got = []
            if case["loss"]:
                other = torch.cat([log_q.gather(1, ids), log_qr], 1)
                t = torch.where(log_p > -math.inf, torch.exp(log_p) * (log_p - other), 0.0).sum(1)
                got.append(t.masked_fill(~there, 0.0))
            if case["grad"]:
                target = torch.exp(log_q - log_qr + log_p[:, -1:]) if s["tail"] is not None else torch.zeros_like(log_q)
                target.scatter_(1, ids, torch.exp(log_p[:, :-1]))
                g = (torch.exp(log_q) - target) * (s["weights"].reshape(-1, 1)[sl].to(D) / tau)
                got.append(g.masked_fill(~there[:, None], 0.0))
            parts.append(tuple(got))
    out = [torch.cat(p).reshape(B, T, *p[0].shape[1:]) for p in zip(*parts)]
    if case["op"] == "process":
        return out[0]
    if case["op"] == "top":
        return [out[0], None, out[1]]
    return out
