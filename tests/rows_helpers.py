"""The operators on rows of scores from their definitions, in 64 bits on the
CPU, with the bounds that their tests use.

Bounds.  EPS = 2^-24 is half a step of fp32.  A row's log-sum m + log(sum of
2^((x - m) log2 e)): an exponent is off by 2 EPS |x - m| and the exponential by
2 EPS, which over a softmax (mean |x - m| <= log W <= 13) is at most 30 EPS of
the sum; a lane adds at most W/64 terms, one rounding each, and 16 roundings
join the lanes; m + log rounds once at the size of both.  A score itself takes
four roundings (a product or quotient, two differences, a sum).  Together at
most EPS (8 X + W/64 + 64), X the largest finite |score| of the row, with
log W below 13 in the constant."""
from __future__ import annotations

import math

import torch

EPS = 2.0 ** -24
LARGEST = float(torch.finfo(torch.float32).max)
TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def clean(x):
    return torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x).clamp(max=LARGEST)


def log_sum(x):
    """Over the last axis, -inf for a row that holds nothing."""
    m = x.amax(-1)
    m0 = torch.where(m > -math.inf, m, torch.zeros_like(m))
    return m0 + torch.log(torch.exp(x - m0[..., None]).sum(-1))


def size(x):
    """The largest finite magnitude of each row."""
    return torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)


def score_bound(x):
    return EPS * (8 * size(x) + x.shape[-1] / 64 + 64)


def frames(lengths, B, T):
    n = torch.full((B,), T) if lengths is None else lengths.cpu().long().clamp(0, T)
    return torch.arange(T)[None] < n[:, None]


def allowed(mask, B, T, W):
    """[B, T, W] truth values of bit words [words], [B, words] or [B, T, words]."""
    m = mask.cpu().to(torch.int64) & 0xFFFFFFFF
    m = m.expand(B, T, m.shape[-1]) if m.dim() != 2 else m[:, None].expand(B, T, m.shape[-1])
    c = torch.arange(W)
    return ((m[..., c // 32] >> (c % 32)) & 1).bool()


def words_of(ok):
    """int32 bit words of truth values [..., W]."""
    W = ok.shape[-1]
    pad = torch.zeros((*ok.shape[:-1], -W % 32), dtype=torch.bool)
    b = torch.cat([ok, pad], -1).reshape(*ok.shape[:-1], -1, 32).to(torch.int64)
    w = (b << torch.arange(32)).sum(-1)
    return torch.where(w >= 2 ** 31, w - 2 ** 32, w).to(torch.int32)


def process(logits, history=None, history_lengths=None, penalties=None, scalars=(1.0, 0.0, 0.0), bias=None, mask=None,
            normalize=True):
    x = clean(logits.cpu().double())
    B, T, W = x.shape
    if history is not None:
        n = torch.zeros((B, W), dtype=torch.float64)
        for b in range(B):
            h = history[b].cpu().long()
            if history_lengths is not None:
                h = h[:max(0, int(history_lengths[b]))]
            h = h[(h >= 0) & (h < W)]
            n[b] = torch.bincount(h, minlength=W).double()
        pen = penalties.cpu().double() if penalties is not None else torch.tensor([scalars], dtype=torch.float32).double().expand(B, 3)
        for b in range(B):
            r, pre, fre = pen[b].tolist()
            seen = torch.where(x[b] > 0, x[b] / r, x[b] * r) - fre * n[b] - pre
            x[b] = torch.where(n[b] > 0, seen, x[b])
    if bias is not None:
        bb = bias.cpu().double()
        x = x + (bb if bb.dim() == 1 else bb[:, None])
    x = clean(x)
    # the scores are fp32's: a sum from half a step beyond its lowest number on is -inf
    x = torch.where(x <= -LARGEST * (1 + EPS / 2), torch.full_like(x, -math.inf), x)
    if mask is not None:
        x = torch.where(allowed(mask, B, T, W), x, torch.full_like(x, -math.inf))
    tol = score_bound(x)
    if normalize:
        total = log_sum(x)
        x = x - torch.where(total > -math.inf, total, torch.zeros_like(total))[..., None]
    return x, tol


def top(logits, k, lengths=None, temperature=1.0):
    x = clean(logits.cpu().double())
    B, T, W = x.shape
    v, i = torch.sort(x, dim=-1, descending=True, stable=True)
    there = frames(lengths, B, T)
    if k < W:
        rest = v[..., k:] / temperature
        tail, tol = log_sum(rest), score_bound(rest)
    else:
        tail, tol = torch.full((B, T), -math.inf, dtype=torch.float64), torch.zeros((B, T), dtype=torch.float64)
    values, ids = v[..., :k].clone(), i[..., :k].to(torch.int32)
    values[~there], ids[~there], tail[~there] = -math.inf, -1, -math.inf
    return values, ids, tail, tol


def distill(student, values, ids, tail=None, lengths=None, temperature=1.0, weights=None):
    """(loss, its bound, gradient, its bound without the rounding to the student's type)."""
    B, T, W = student.shape
    k = values.shape[-1]
    s = 1.0 / temperature
    there = frames(lengths, B, T)
    loss, loss_tol = torch.zeros((B, T), dtype=torch.float64), torch.zeros((B, T), dtype=torch.float64)
    grad, grad_tol = torch.zeros((B, T, W), dtype=torch.float64), torch.zeros((B, T, W), dtype=torch.float64)
    student, values, ids = student.cpu().double(), values.cpu().double(), ids.cpu().long()
    for b in range(B):
        for t in range(T):
            if not there[b, t]:
                continue
            x = student[b, t] * s
            v = clean(values[b, t])
            real = (ids[b, t] >= 0) & (ids[b, t] < W) & (v > -math.inf)
            u = (v * s).clamp(max=LARGEST)[real]
            at = ids[b, t][real]
            r = -math.inf if tail is None else float(clean(tail[b, t].cpu().double()))
            both = torch.cat([u, torch.tensor([r], dtype=torch.float64)])
            total = float(log_sum(both))
            if total == -math.inf or (x.max() == -math.inf and not torch.isnan(x).any()):
                continue
            p = torch.exp(both - total)
            P = torch.zeros(W, dtype=torch.float64).index_add_(0, at, p[:-1])
            listed = torch.zeros(W, dtype=torch.bool)
            listed[at] = True
            lse = x.max() + torch.log(torch.exp(x - x.max()).sum())
            log_q = x - lse
            rest = torch.where(listed, torch.full_like(x, -math.inf), x)
            rest_sum = log_sum(rest)
            some = P > 0
            parts = torch.where(some, P * (torch.log(torch.where(some, P, torch.ones_like(P))) - log_q), torch.zeros_like(P))
            pr = float(p[-1])
            last = pr * ((r - total) - (rest_sum - lse)) if pr > 0 else torch.zeros((), dtype=torch.float64)
            loss[b, t] = parts.sum() + last
            X = float(max(size(x), size(both)))
            unit = EPS * (16 * X + W / 32 + 128)
            loss_tol[b, t] = unit * (1 + float(parts.abs().sum() + abs(last)))
            q = torch.exp(log_q)
            in_rest = pr * torch.exp(rest - rest_sum) if rest_sum > -math.inf else torch.zeros_like(q)
            w = float(weights[b, t]) if weights is not None else 1.0
            grad[b, t] = torch.where(listed, q - P, q - in_rest) * w * s
            grad_tol[b, t] = unit * abs(w) * s * (q + P + in_rest) + 1e-37
    return loss, loss_tol, grad, grad_tol


def rounded_bound(grad, tol, kind):
    """The bound with the one rounding to the gradient's type (fp16's smallest step is 2^-24)."""
    half = torch.finfo(TYPES[kind]).eps / 2
    tiny = {"fp32": 2.0 ** -150, "fp16": 2.0 ** -25, "bf16": 2.0 ** -134}[kind]
    return tol * (1 + half) + grad.abs() * half + tiny


def near(got, want, tol, what=""):
    """Equal infinities and NaN, and all else within the bound."""
    got, want = got.detach().cpu().double(), want.double()
    tol = tol.double().expand_as(want) if tol.dim() == want.dim() else tol.double()[..., None].expand_as(want)
    assert got.shape == want.shape, f"{what}: {tuple(got.shape)} and {tuple(want.shape)}"
    odd = ~torch.isfinite(want)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    bad = torch.where(odd, ~same, ~((got - want).abs() <= tol))
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off, first at {at}: {got[at]} for {want[at]} (bound {tol[at]:.3g})")
