"""Every kernel of the operators on rows of scores against the definitions in
64 bits (bounds: rows_helpers), at both ends of the lengths that it takes.

Long rows are compared with the definition once for each of 16 different rows
and lists, regular and odd ones; a call has many of each, in other places of
the batch, and these have to have the same bits."""
import functools
import math

import pytest
import torch

import paper_2508_07315_amd as P
import rows_helpers as R
from rows_calls import DISTILL, KINDS, PROCESS, TOP, of_kind
from test_gpu_rows import dev, gen, scores

pytestmark = pytest.mark.gpu
INF = math.inf
DIFFERENT = 16
BITS = {torch.float32: torch.int32, torch.int32: torch.int32, torch.float16: torch.int16, torch.bfloat16: torch.int16}


def calls(of):
    return [(kind, *c) for kind in KINDS for c in of_kind(of, kind)]


def lengths_of(B, T):
    """T and what lies around it, 0 and 1 among them."""
    return torch.tensor([(T, T - 1, 0, T + 3, 1, T)[b % 6] for b in range(B)], dtype=torch.int32)


def spread(rows, B, T):
    """[B, T, ...] of the different rows in turn."""
    return rows[torch.arange(B * T, device=rows.device) % len(rows)].reshape(B, T, *rows.shape[1:])


def one_of_each(got, lengths, behind, what):
    """The result of each different row, where all of a kind have the same bits; those behind the lengths have `behind`."""
    B, T = got.shape[:2]
    there = R.frames(lengths, B, T).reshape(-1).to(got.device)
    flat = got.reshape(B * T, *got.shape[2:])
    bits = flat.contiguous().view(BITS[got.dtype])
    kind = torch.arange(B * T, device=got.device) % DIFFERENT
    assert (flat[~there] == behind).all(), f"{what}: frames behind the lengths"
    first = []
    for d in range(DIFFERENT):
        at = (there & (kind == d)).nonzero().flatten()
        if len(at) == 0:
            first.append(None)
            continue
        assert (bits[at] == bits[at[0]]).all(), f"{what}: row {d} differs from place to place"
        first.append(flat[at[0]].cpu())
    return first


def near_each(first, want, tol, what):
    seen = [d for d, f in enumerate(first) if f is not None]
    assert len(seen) > DIFFERENT // 2, "too few of the different rows are there"
    R.near(torch.stack([first[d] for d in seen]), want[seen], tol[seen], what)


def in_a_buffer(x, odd):
    """The same values where a caller has them: rows of a wider buffer, or as they are."""
    if not odd:
        return x.to(dev())
    B, T, W = x.shape
    buf = torch.full((B, T, W + 3), 9.0, dtype=x.dtype, device=dev())
    buf[:, :, 1:W + 1] = x.to(dev())
    return buf[:, :, 1:W + 1]


# ------------------------------------------------------------------- process

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,T,W,H,normalize", PROCESS)
def test_process(kind, B, T, W, H, normalize):
    g, d = gen(B + T + W), dev()
    x = scores(B, T, W, kind, W + H, order="slice")
    lengths = lengths_of(B, T) if T > 1 else None
    kw, ref = dict(normalize=normalize), dict(normalize=normalize)
    if H:
        h = torch.randint(-1, W + 1, (B, H), generator=g, dtype=torch.int32)
        h[:, ::4] = W - 1
        hl = torch.randint(0, H + 2, (B,), generator=g, dtype=torch.int32)
        pen = torch.rand((B, 3), generator=g) + 0.5
        kw.update(history=h.to(d), history_lengths=hl.to(d), penalties=pen.to(d))
        ref.update(history=h, history_lengths=hl, penalties=pen)
    bias = torch.randn((B, W), generator=g)
    # a bit of a frame and one of its label: some frames, and so some rows of a workgroup, are left with nothing
    words = R.words_of(torch.rand((B, 1, W), generator=g) < 0.7).expand(B, T, -1).clone()
    words[:, 1::3] = 0
    if T == 1:
        words[1::3] = 0
    kw.update(bias=bias.to(d), mask=words.to(d))
    ref.update(bias=bias, mask=words)
    want, tol = R.process(x, **ref)
    ln = None if lengths is None else lengths.to(d)
    out = torch.full((B, T, W), 123.0, device=d)
    P.process_logits(x, ln, out=out, **kw)
    there = R.frames(lengths, B, T)
    R.near(out[there.to(d)], want[there], tol[there], f"{kind} {B} {T} {W} {H}")
    assert (out[~there.to(d)] == 123.0).all(), "rows behind the lengths were written"
    again = torch.full((B, T, W), 123.0, device=d)
    P.process_logits(x, ln, out=again, **kw)
    assert torch.equal(again, out)
    if kind == "fp32":
        y = x.contiguous()
        P.process_logits(y, ln, out=y, **kw)
        assert torch.equal(y[there.to(d)], out[there.to(d)]) and torch.equal(y[~there.to(d)], x[~there.to(d)])


# ----------------------------------------------------------------------- top

@functools.lru_cache(maxsize=2)
def top_rows(W):
    """16 rows: random ones, and rows of ties, of order, of nothing, of a far tail."""
    x = torch.randn((DIFFERENT, W), generator=gen(W)) * 2.0
    x[1, -1] += 9.0
    c = torch.arange(W)
    x[2] = (c % 7 == 3).float()
    x[3] = -INF
    x[4] = -INF
    x[4, W // 2] = 1.0
    x[5] = ((c // 40) % 1000).float()
    x[6] = math.nan
    x[7, ::2] = math.nan
    x[8] = -500.0
    x[8, W // 3] = 500.0
    x[9] = (c % 1000).float()
    x[10] = -(c % 1000).float()
    x[11] = 0.0
    x[12, W - 5:] = INF
    x[13, :W // 2] = -INF
    x[14] = torch.where(c % 2 == 0, -0.0, 0.0)
    x[15, W // 2:] += 20.0
    return x


@pytest.mark.parametrize("kind,B,T,W,k", calls(TOP))
def test_top(kind, B, T, W, k):
    x = top_rows(W).to(R.TYPES[kind])
    lengths, temperature, what = lengths_of(B, T), 2.0, f"{kind} {B} {T} {W} {k}"
    want_v, want_i, want_t, tol = (a[0] for a in R.top(x[None], k, temperature=temperature))
    full = in_a_buffer(spread(x, B, T), W % 2)
    got = P.top_logits(full, k, lengths.to(dev()), temperature=temperature)
    for name, a, w, behind in zip(("values", "ids"), got, (want_v, want_i), (-INF, -1)):
        for d, f in enumerate(one_of_each(a, lengths, behind, f"{what}: {name}")):
            assert f is None or torch.equal(f.double(), w[d].double()), f"{what}: {name} of row {d}"
    near_each(one_of_each(got[2], lengths, -INF, f"{what}: tail"), want_t, tol, f"{what}: tail")
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(P.top_logits(full, k, lengths.to(dev()), temperature=temperature), got)), what


# ------------------------------------------------------------------- distill

def distill_rows(W, k):
    """16 students and their teachers' lists: regular ones, odd lists, odd students."""
    g = gen(W + k)
    t = torch.randn((DIFFERENT, W), generator=g) * 2.0
    t[:, -1] += 3.0
    v, ids = torch.topk(t, k, dim=-1)
    tail = torch.logsumexp(t.scatter(1, ids, -INF) / 2.0, -1)
    ids = ids.to(torch.int32)
    x = torch.randn((DIFFERENT, W), generator=g) * 2.0
    x[:, -1] += 4.0
    ids[1, :5] = torch.tensor([3, 3, W - 1, 3, W - 1], dtype=torch.int32)          # twice and three times
    ids[2, :4] = torch.tensor([-1, W, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)   # no labels
    ids[3] = -1                                                                   # no entry, but a tail
    ids[4], tail[4] = -1, -INF                                                    # nothing
    v[5, :3] = torch.tensor([-INF, math.nan, INF])
    v[6], tail[6] = -200.0, 0.0                                                   # all of the mass beside the list
    tail[7] = -INF
    ids[8] = torch.arange(k, dtype=torch.int32) * (W // k)                        # at even distances, labels of each vector
    ids[8, 0] = W - 1
    x[9] = -INF
    x[10, int(ids[10, 0])] = -INF                                                 # a listed label is barred
    others = torch.ones(W, dtype=torch.bool)
    others[ids[11].long()] = False
    x[11, others] = -INF                                                          # all others are barred
    x[12, others] = -150.0
    x[13, W // 2] = math.nan
    x[14, W // 2] = INF
    x[15, :W // 2] = -INF
    return x, v, ids, tail


@pytest.mark.parametrize("kind,B,T,W,k", calls(DISTILL))
def test_distill(kind, B, T, W, k):
    x, v, ids, tail = distill_rows(W, k)
    x = x.to(R.TYPES[kind])
    w = torch.rand((DIFFERENT,), generator=gen(k)) + 0.5
    loss_want, loss_tol, grad_want, grad_tol = (a[0] for a in R.distill(x[None], v[None], ids[None], tail[None], temperature=2.0, weights=w[None]))
    lengths, what, d = lengths_of(B, T), f"{kind} {B} {T} {W} {k}", dev()
    args = [in_a_buffer(spread(x, B, T), W % 2), *(spread(a.to(d), B, T) for a in (v, ids, tail)), lengths.to(d)]
    kw = dict(temperature=2.0, weights=spread(w.to(d), B, T))
    loss, grad = P.distill(*args, **kw)
    near_each(one_of_each(loss, lengths, 0.0, f"{what}: loss"), loss_want, loss_tol, f"{what}: loss")
    near_each(one_of_each(grad, lengths, 0.0, f"{what}: gradient"), grad_want, R.rounded_bound(grad_want, grad_tol, kind), f"{what}: gradient")

    def same(a, b):
        return torch.equal(a.view(BITS[a.dtype]), b.view(BITS[b.dtype]))
    for _ in range(3):
        assert all(same(a, b) for a, b in zip(P.distill(*args, **kw), (loss, grad))), what
    assert same(P.distill(*args, **kw, want_grad=False)[0], loss), what
    buf = torch.full((B, T, W + 5), 9.0, dtype=x.dtype, device=d)                 # the gradient in rows of a wider buffer
    P.distill(*args, **kw, want_loss=False, grad=buf[:, :, 3:W + 3])
    assert same(buf[:, :, 3:W + 3].contiguous(), grad), what
    assert (buf[:, :, :3] == 9.0).all() and (buf[:, :, W + 3:] == 9.0).all(), what


def test_small_temperatures():
    """The least that is accepted: what is not the largest is infinitely far, nothing is NaN."""
    for W in (40, 2000, 9300, 150000):
        x = scores(2, 3, W, "fp32", W)
        v, ids, tail = P.top_logits(x, 2, temperature=4.3e-39)
        assert torch.equal(ids.cpu(), R.top(x, 2)[1]) and not torch.isnan(tail).any()
        loss, grad = P.distill(x, v, ids, tail, temperature=4.3e-39)
        assert not torch.isnan(loss).any() and not torch.isnan(grad).any()


def test_tails_that_are_no_number():
    """NaN counts as -inf, +inf as the largest number."""
    for B, T, W in ((2, 3, 40), (300, 4, 33), (2, 3, 2500), (2, 3, 9300), (1, 2, 150000)):
        x = scores(B, T, W, "fp32", W)
        v, ids, tail = P.top_logits(x, 4)
        for odd, plain in ((math.nan, -INF), (INF, R.LARGEST)):
            a, b = tail.clone(), tail.clone()
            a[0, 1], b[0, 1] = odd, plain
            assert all(torch.equal(p, q) for p, q in zip(P.distill(x * 0.5, v, ids, a), P.distill(x * 0.5, v, ids, b)))
