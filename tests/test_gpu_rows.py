"""The operators on rows of scores on the GPU against their definitions in 64
bits (bounds: rows_helpers)."""
import math

import pytest
import torch

import paper_2508_07315_amd as P
import rows_helpers as R

pytestmark = pytest.mark.gpu
INF = math.inf


def dev():
    assert torch.cuda.is_available(), "GPU test without a GPU"
    return torch.device("cuda:0")


def gen(seed):
    return torch.Generator().manual_seed(seed)


def scores(B, T, W, kind, seed, spread=2.0, order="btw"):
    """[B, T, W] scores on the device, in one of the orders a caller has them in."""
    x = torch.randn((B, T, W), generator=gen(seed)) * spread
    x[..., -1] += 4.0
    x = x.to(R.TYPES[kind])
    d = dev()
    if order == "btw":
        return x.to(d)
    if order == "tbw":                               # frames outside, as recurrent models give them
        return x.transpose(0, 1).contiguous().to(d).transpose(0, 1)
    if order == "slice":                             # rows of a wider buffer, the first one off its start
        buf = torch.full((B, T + 1, W + 3), 7.0, dtype=x.dtype, device=d)
        buf[:, :T, 1:W + 1] = x.to(d)
        return buf[:, :T, 1:W + 1]
    if order == "repeat":                            # one utterance's rows for all
        return x[:1].to(d).expand(B, T, W)
    raise ValueError(order)


WIDTHS = [1, 2, 5, 33, 64, 255, 1025, 2049, 4097, 9999, 40001, 131073]
ORDERS = ["btw", "tbw", "slice", "repeat"]
KINDS = ["fp32", "fp16", "bf16"]


def pick(i, values):
    return values[i % len(values)]


# ------------------------------------------------------------------- process

def process_case(B, T, W, kind, seed, H=0, bias="none", mask="none", order="btw", lengths=None, normalize=True,
                 penalties=True):
    d, g = dev(), gen(seed + 1)
    x = scores(B, T, W, kind, seed, order=order)
    kw = dict(normalize=normalize)
    ref = dict(normalize=normalize)
    if H:
        h = torch.randint(-1, W + 2, (B, H), generator=g, dtype=torch.int32)
        h[:, ::3] = int(W // 2)                      # one label over and over
        hl = torch.randint(0, H + 3, (B,), generator=g, dtype=torch.int32) - 1
        kw.update(history=h.to(d), history_lengths=hl.to(d))
        ref.update(history=h, history_lengths=hl)
        if penalties:
            p = torch.rand((B, 3), generator=g) + 0.6
            p[0] = torch.tensor([1.5, -0.5, 0.25])
            kw["penalties"], ref["penalties"] = p.to(d), p
        else:
            kw.update(repetition=1.25, presence=0.5, frequency=0.125)
            ref["scalars"] = (1.25, 0.5, 0.125)
    if bias != "none":
        b = torch.randn((W,) if bias == "shared" else (B, W), generator=g)
        kw["bias"], ref["bias"] = b.to(d), b
    if mask != "none":
        shape = {"all": (W,), "row": (B, W), "frame": (B, T, W)}[mask]
        ok = torch.rand(shape, generator=g) < 0.6
        if mask != "all":
            ok[0] = False                            # a row in which nothing is allowed
        m = R.words_of(ok)
        if W % 32:
            m[..., -1] |= -1 << (W % 32)             # bits behind the last label mean nothing
        kw["mask"], ref["mask"] = m.to(d), m
    want, tol = R.process(x, **ref)
    out = torch.full((B, T, W), 123.0, device=d)
    got = P.process_logits(x, None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=d), out=out, **kw)
    torch.cuda.synchronize()
    there = R.frames(None if lengths is None else torch.tensor(lengths), B, T)
    R.near(got[there.to(d)], want[there], tol[there], f"process W={W} {kind}")
    assert (got[~there.to(d)] == 123.0).all(), "rows behind the lengths were written"


@pytest.mark.parametrize("i,W", list(enumerate(WIDTHS)))
@pytest.mark.parametrize("kind", KINDS)
def test_process_widths(i, W, kind):
    i += KINDS.index(kind)
    B, T = (3, 5) if W < 20000 else (2, 3)
    process_case(B, T, W, kind, 100 + i, H=pick(i, [0, 7, 300]), bias=pick(i // 2, ["none", "shared", "row"]),
                 mask=pick(i // 3, ["none", "row", "frame", "all"]), order=pick(i, ORDERS),
                 lengths=pick(i, [None, [T, 0, T + 4][:B], [2, -1, 1][:B]]), normalize=i % 5 != 4, penalties=i % 2 == 0)


@pytest.mark.parametrize("B,T,W,H", [(1, 1, 1025, 24), (37, 1, 1025, 9), (5, 1, 32003, 20000), (1, 1, 131072, 1), (9, 130, 33, 5),
                                     (2, 700, 100, 64), (300, 1, 515, 3), (1100, 1, 1025, 6), (700, 3, 65, 2),
                                     (70, 1, 40001, 5), (150, 1, 30003, 3), (2, 80, 30003, 40000)])
def test_process_steps_and_utterances(B, T, W, H):
    process_case(B, T, W, "bf16", B + W, H=H, bias="row", mask="row")


def test_process_long_history_of_one_label():
    """70,000 times the same label (more than 16 bits count), in a small and a large row."""
    for W in (40, 50001):
        x = scores(1, 1, W, "fp32", 5)
        h = torch.full((1, 70000), W - 2, dtype=torch.int32)
        want, tol = R.process(x, history=h, scalars=(1.0, 0.0, 0.001), normalize=False)
        got = P.process_logits(x, history=h.to(dev()), frequency=0.001, normalize=False)
        # the penalty itself, 70 of 0.001f * 70000, is one rounding more
        R.near(got, want, tol + 70 * R.EPS, f"W={W}")


def test_process_odd_values():
    """NaN, infinities, the type's lowest value as a bias, and rows that nothing is left of."""
    low = -R.LARGEST
    x = torch.tensor([[1.0, math.nan, 2.0, -INF, 0.5], [INF, 1.0, INF, -INF, math.nan], [-INF] * 5, [math.nan] * 5,
                      [1.0, 2.0, 3.0, 4.0, 5.0], [low, low, low, low, low], [R.LARGEST] * 5, [0.0, -0.0, 0.0, -0.0, 1.0]])
    bias = torch.zeros(8, 5)
    bias[4] = torch.tensor([low, 0.0, low, low, 0.0])
    bias[5] = low
    bias[0, 3], bias[0, 4], bias[1, 0] = INF, -INF, -INF
    bias[6, 0] = R.LARGEST
    x = x[:, None]
    for normalize in (True, False):
        want, _ = R.process(x, bias=bias, normalize=normalize)
        # a difference beyond fp32's largest number is infinite
        want = torch.where(want.abs() >= 2.0 ** 128 * (1 - 2.0 ** -25), torch.sign(want) * INF, want)
        got = P.process_logits(x.to(dev()), bias=bias.to(dev()), normalize=normalize)
        R.near(got, want, 1e-5 * (1 + torch.where(torch.isfinite(want), want.abs(), 0.0)), f"normalize={normalize}")
        assert not torch.isnan(got).any()


def test_process_in_place():
    for W in (33, 1025, 5000, 70001):
        x = scores(3, 4, W, "fp32", W)
        want = P.process_logits(x)
        y = x.clone()
        got = P.process_logits(y, out=y)
        assert got.data_ptr() == y.data_ptr()
        assert torch.equal(got, want)


def test_process_default_is_log_softmax():
    x = scores(4, 6, 1025, "fp16", 3, order="tbw")
    want, tol = R.process(x)
    R.near(P.process_logits(x), want, tol)


# ----------------------------------------------------------------------- top

def top_case(x, k, lengths=None, temperature=1.0, what=""):
    d = dev()
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    want_v, want_i, want_t, tol = R.top(x, k, ln, temperature)
    v, i, t = P.top_logits(x, k, None if ln is None else ln.to(d), temperature=temperature)
    torch.cuda.synchronize()
    assert torch.equal(i.cpu(), want_i), f"{what}: ids"
    assert torch.equal(v.cpu().double(), want_v), f"{what}: values"
    R.near(t, want_t, tol, f"{what}: tail")


@pytest.mark.parametrize("i,W", list(enumerate(WIDTHS)))
@pytest.mark.parametrize("kind", KINDS)
def test_top_widths(i, W, kind):
    B, T = (3, 5) if W < 20000 else (2, 2)
    for j, k in enumerate([1, 2, 16, 64, 65, 128]):
        if k <= W:
            x = scores(B, T, W, kind, 200 + i + j, order=pick(i + j, ORDERS))
            top_case(x, k, pick(i + j, [None, [T, 0, T + 4][:B], [2, -1, 1][:B]]), pick(j, [1.0, 0.5, 3.0]),
                     f"W={W} k={k} {kind}")
    if W <= 128:
        top_case(scores(B, T, W, kind, 7), W, what=f"all of {W}")


@pytest.mark.parametrize("W", [40, 1025, 5003, 70000, 262144])
@pytest.mark.parametrize("k", [1, 5, 40])
def test_top_of_ties(W, k):
    """Rows of one value, of two, ascending, descending, in blocks, of nothing."""
    c = torch.arange(W).float()
    r = torch.zeros(9, 1, W)
    r[1] = (c % 7 == 3).float()
    r[2] = c
    r[3] = -c
    r[4] = -INF
    r[5] = -INF
    r[5, 0, W // 3] = 1.0
    r[6] = (c >= W - 30).float() * 2.0
    r[7] = torch.where(c % 2 == 0, -0.0, 0.0)
    r[8] = math.nan
    r[8, 0, W - 1] = INF
    top_case(r.to(dev()), k, what=f"W={W} k={k}")


@pytest.mark.parametrize("B,T,W,k", [(1, 1, 262144, 128), (1, 3, 262143, 100), (40, 1, 50001, 64), (1, 300, 2000, 8), (700, 1, 129, 128)])
def test_top_sizes(B, T, W, k):
    top_case(scores(B, T, W, "bf16", W + k), k, what=f"B={B} T={T} W={W} k={k}")


@pytest.mark.parametrize("W,k", [(33, 32), (64, 1), (1025, 16), (1279, 32), (1280, 5), (2303, 32), (2304, 7)])
@pytest.mark.parametrize("kind", KINDS)
def test_top_many_rows(W, k, kind):
    """Enough rows for the form that gives each a wave, with rows of ties, of nothing and of a far tail among them."""
    x = torch.randn((9, 130, W), generator=gen(W)) * 2.0
    c = torch.arange(W).float()
    x[1, :, :] = (c % 7 == 3).float()
    x[2, 5], x[2, 6] = -INF, -INF
    x[2, 6, W // 2] = 1.0
    x[3, 7] = c // 40
    x[3, 8] = math.nan
    x[3, 9, ::2] = math.nan
    x[3, 10] = -500.0
    x[3, 10, W // 3] = 500.0
    top_case(x.to(R.TYPES[kind]).to(dev()), k, [130, 7, 100, 130, 0, 1, 130, 129, 64], 2.0, f"W={W} k={k} {kind}")


def test_top_of_the_longest_spans():
    """A row whose halves, in whole words, are as long as a workgroup holds: the largest labels are the last of each."""
    W = 139255
    x = torch.randn((1, 2, W), generator=gen(3))
    x[..., 69500:69700] += 10.0
    x[..., -100:] += 10.0
    top_case(x.to(dev()), 128, what=f"W={W}")


def test_top_tail_far_below():
    """What is left may lie far below the list: its log-sum stays finite."""
    x = torch.full((1, 2, 900), -300.0)
    x[0, 0, 5], x[0, 1, 899] = 400.0, 0.0
    top_case(x.to(dev()), 1)
    top_case(x.to(dev()), 3)


# ------------------------------------------------------------------- distill

def teacher(B, T, W, k, seed, temperature=1.0, tail=True):
    x = torch.randn((B, T, W), generator=gen(seed)) * 2.0
    x[..., -1] += 3.0
    v, i = torch.topk(x, k, dim=-1)
    rest = torch.logsumexp(x.scatter(2, i, -INF) / temperature, -1) if tail else None
    return v.contiguous(), i.to(torch.int32).contiguous(), rest


def distill_case(x, v, i, tail, lengths=None, temperature=1.0, weights=None, what="", kind="fp32", grad=None):
    d = dev()
    ln = None if lengths is None else torch.tensor(lengths, dtype=torch.int32)
    loss, loss_tol, want, tol = R.distill(x, v, i, tail, ln, temperature, weights)
    args = (x, v.to(d), i.to(d), None if tail is None else tail.to(d), None if ln is None else ln.to(d))
    kw = dict(temperature=temperature, weights=1.0 if weights is None else weights.to(d))
    got_loss, got = P.distill(*args, **kw, grad=grad)
    torch.cuda.synchronize()
    R.near(got_loss, loss, loss_tol, f"{what}: loss")
    R.near(got, want, R.rounded_bound(want, tol, kind), f"{what}: gradient")
    # each alone is the same
    assert torch.allclose(P.distill(*args, **kw, want_grad=False)[0], got_loss, rtol=0, atol=0, equal_nan=True)
    assert torch.allclose(P.distill(*args, **kw, want_loss=False)[1], got, rtol=0, atol=0, equal_nan=True)
    return got_loss, got


@pytest.mark.parametrize("i,W", list(enumerate(WIDTHS)))
@pytest.mark.parametrize("kind", KINDS)
def test_distill_widths(i, W, kind):
    B, T = (3, 4) if W < 20000 else (2, 2)
    i += KINDS.index(kind)
    for j, k in enumerate([1, 8, 64, 128]):
        if k > W:
            continue
        temperature = pick(i + j, [1.0, 2.0, 0.7])
        v, ids, tail = teacher(B, T, W, k, 300 + i + j, temperature, tail=(i + j) % 3 != 0)
        w = torch.rand((B, T), generator=gen(i)) + 0.5 if j % 2 else None
        distill_case(scores(B, T, W, kind, 400 + i + j, order=pick(i + j, ORDERS)), v, ids, tail,
                     pick(i + j, [None, [T, 0, T + 4][:B], [2, -1, 1][:B]]), temperature, w, f"W={W} k={k} {kind}", kind)


@pytest.mark.parametrize("B,T,W,k", [(1, 1, 262144, 128), (260, 1, 700, 4), (1, 300, 1025, 16), (30, 1, 20001, 50),
                                     (300, 4, 33, 5), (2, 520, 1025, 128), (1030, 1, 2303, 16),
                                     (130, 1, 9216, 20), (2, 65, 40959, 128), (1, 140, 81921, 64), (128, 1, 139263, 9), (70, 1, 40001, 16)])
def test_distill_sizes(B, T, W, k):
    v, ids, tail = teacher(B, T, W, k, W)
    distill_case(scores(B, T, W, "bf16", W + 1), v, ids, tail, what=f"B={B} T={T} W={W}", kind="bf16")


ODD_ROWS = [(50, 1), (1025, 1), (1025, 130), (2303, 130), (6000, 1), (90000, 1), (9300, 17),
            (60001, 17)]                                   # labels, times the 8 rows


@pytest.mark.parametrize("W,times", ODD_ROWS)
def test_distill_odd_lists(W, times):
    """Ids twice and three times, ids out of range, empty lists, values of -inf and NaN, all of the mass in the tail."""
    x = scores(8, 1, W, "fp32", W)
    v, ids, tail = teacher(8, 1, W, 6, W + 1)
    ids[0, 0] = torch.tensor([3, 3, 9, 3, 9, 1])
    ids[1, 0] = torch.tensor([-1, W, 2 ** 31 - 1, -2 ** 31, W - 1, 0])
    ids[2, 0] = -1                                    # no entry, but a tail
    ids[3, 0], tail[3, 0] = -1, -INF                  # nothing
    v[4, 0] = torch.tensor([1.0, -INF, math.nan, 0.5, -INF, 2.0])
    v[5, 0] = -INF
    v[6, 0], tail[6, 0] = -200.0, 0.0                 # the list holds next to nothing
    tail[7, 0] = -INF
    x, v, ids, tail = (a.repeat(times, *[1] * (a.dim() - 1)) for a in (x, v, ids, tail))
    loss, grad = distill_case(x, v, ids, tail, what=f"W={W}")
    assert loss[3, 0] == 0 and (grad[3] == 0).all()


@pytest.mark.parametrize("W,times", ODD_ROWS)
def test_distill_odd_students(W, times):
    """Barred labels, rows of -inf, peaks that leave the rest far below, NaN and +inf."""
    x = scores(8, 1, W, "fp32", W)
    v, ids, tail = teacher(8, 1, W, 6, W + 1)
    x[0] = -INF                                       # no distribution: loss and gradient 0
    x[1, 0, int(ids[1, 0, 0])] = -INF                 # a listed label is barred: loss +inf
    others = torch.ones(W, dtype=torch.bool)
    others[ids[2, 0].long()] = False
    x[2, 0, others.to(x.device)] = -INF               # the rest is barred: +inf through the tail
    x[3, 0, others.to(x.device)] = -150.0             # the rest lies far below
    x[4, 0, int(ids[4, 0, 0])] += 250.0
    x[5, 0, W // 2] = math.nan
    x[6, 0, W // 2] = INF
    x[7, 0, :W // 2] = -INF
    x, v, ids, tail = (a.repeat(times, *[1] * (a.dim() - 1)) for a in (x, v, ids, tail))
    loss, grad = distill_case(x, v, ids, tail, what=f"W={W}")
    assert (loss[0] == 0).all() and (grad[0] == 0).all()
    assert loss[1, 0] == INF and torch.isfinite(grad[1]).all()
    assert loss[2, 0] == INF and torch.isfinite(grad[2]).all()
    assert torch.isnan(loss[5]).all() and torch.isnan(grad[5]).all()


def test_distill_all_labels_listed():
    """k = W: nothing is left, with a tail and without."""
    x = scores(2, 3, 20, "fp32", 1)
    v, ids, _ = teacher(2, 3, 20, 20, 2, tail=False)
    distill_case(x, v, ids, None)
    loss, _ = distill_case(x, v, ids, torch.zeros(2, 3))
    assert (loss == INF).all()


def test_distill_of_itself_is_zero():
    x = scores(2, 9, 1025, "fp32", 4)
    v, ids, tail = P.top_logits(x, 16)
    loss, grad = distill_case(x, v.cpu(), ids.cpu(), tail.cpu())
    assert loss.abs().max() < 1e-5


def test_distill_gradient_layouts():
    """The gradient in rows of a wider buffer, frames outside; what lies between stays."""
    B, T, W = 3, 4, 1025
    for kind in ("fp32", "bf16"):
        v, ids, tail = teacher(B, T, W, 8, 6)
        x = scores(B, T, W, kind, 5)
        buf = torch.full((T, B, W + 5), 9.0, dtype=R.TYPES[kind], device=dev())
        grad = buf.transpose(0, 1)[:, :, 2:W + 2]
        distill_case(x, v, ids, tail, [4, 2, 0], kind=kind, grad=grad)
        assert (buf[:, :, :2] == 9.0).all() and (buf[:, :, W + 2:] == 9.0).all()


def test_distill_gradient_is_the_slope():
    """Against central differences of the 64-bit loss (h = 1e-5: their error is below 1e-8)."""
    x = scores(1, 2, 12, "fp32", 8)
    v, ids, tail = teacher(1, 2, 12, 4, 9, 2.0)
    _, grad = P.distill(x, v.to(dev()), ids.to(dev()), tail.to(dev()), temperature=2.0)
    x64, h = x.cpu().double(), 1e-5
    for t in range(2):
        for c in range(12):
            d = torch.zeros_like(x64)
            d[0, t, c] = h
            up, down = (R.distill(x64 + sign * d, v, ids, tail, temperature=2.0)[0].sum() for sign in (1, -1))
            assert abs(float(grad[0, t, c]) - float(up - down) / (2 * h)) < 2e-6


def test_distill_loss_differentiates():
    """Through torch: reductions whose upstream gradient is broadcast, weighted sums, a student used twice."""
    B, T, W = 3, 5, 130
    lengths = torch.tensor([5, 3, 0], dtype=torch.int32)
    v, ids, tail = teacher(B, T, W, 8, 11, 2.0)
    x = scores(B, T, W, "fp32", 12)
    d = dev()
    args = (v.to(d), ids.to(d), tail.to(d), lengths.to(d), 2.0)
    w = torch.rand((B, T), generator=gen(1))
    for reduce, weights in ((lambda l: l.sum(), torch.ones(B, T)), (lambda l: l.mean(), torch.full((B, T), 1 / (B * T))),
                            (lambda l: (l * w.to(d)).sum(), w), (lambda l: l.t().sum(0).sum(), torch.ones(B, T))):
        leaf = x.clone().requires_grad_()
        reduce(P.distill_loss(leaf, *args)).backward()
        _, _, want, tol = R.distill(x, v, ids, tail, lengths, 2.0, weights)
        R.near(leaf.grad, want, R.rounded_bound(want, tol, "fp32"))
    leaf = x.clone().requires_grad_()
    (P.distill_loss(leaf * 0.5, *args).sum() + P.distill_loss(leaf * 0.5, *args).sum()).backward()
    _, _, want, tol = R.distill(x * 0.5, v, ids, tail, lengths, 2.0)
    R.near(leaf.grad, want, R.rounded_bound(want, tol, "fp32") * 2)
    leaf = x.clone().requires_grad_()
    P.distill_loss(leaf, args[0], args[1]).sum().backward()                       # no tail, no lengths
    _, _, want, tol = R.distill(x, v, ids)
    R.near(leaf.grad, want, R.rounded_bound(want, tol, "fp32"))
    with torch.no_grad():
        assert not P.distill_loss(leaf, *args).requires_grad
    with pytest.raises(RuntimeError, match="once_differentiable|twice"):
        g, = torch.autograd.grad(P.distill_loss(leaf, *args).square().sum(), leaf, create_graph=True)
        g.sum().backward()


# ------------------------------------------------------- together, and in use

def test_from_logits_to_transcripts():
    """A model's 16-bit logits, processed, through the decoders: the same as the decoders on the log-probabilities of
    the definition (rounded to fp32), with the same transcripts and scores within the sum of the frames' bounds."""
    B, T, W = 4, 40, 33
    x = scores(B, T, W, "bf16", 21, spread=3.0, order="tbw")
    lengths = torch.tensor([40, 25, 1, 0], dtype=torch.int32)
    ok = torch.ones(B, W, dtype=torch.bool)
    ok[:, 5:9] = False
    bias = torch.zeros(W)
    bias[W - 1] = -2.0                                # the blank, held back
    want, tol = R.process(x, bias=bias, mask=R.words_of(ok))
    d = dev()
    lp = P.process_logits(x, lengths.to(d), bias=bias.to(d), mask=R.words_of(ok).to(d))
    for decode in (lambda s: P.decode(s, lengths.to(d), 8, beta=0.5), lambda s: P.ctcbeam_greedy_decode(s, lengths.to(d))[:3]):
        tok, ln, sc = decode(lp)
        tok2, ln2, sc2 = decode(want.float().to(d))
        assert torch.equal(tok, tok2) and torch.equal(ln, ln2)
        assert not ((tok >= 5) & (tok < 9)).any()
        assert ((sc - sc2).abs().cpu() <= tol.max() * T + 1e-4).all()


def test_from_teacher_to_gradient():
    """The teacher's list taken from its logits, and the student's loss against the divergence over all labels of the
    coarse distributions: the same labels, one bucket for the others."""
    B, T, W, k = 3, 6, 1025, 16
    d = dev()
    lengths = torch.tensor([6, 4, 1], dtype=torch.int32, device=d)
    big, small = scores(B, T, W, "bf16", 31), scores(B, T, W, "bf16", 32)
    v, ids, tail = P.top_logits(big, k, lengths, temperature=2.0)
    leaf = small.clone().requires_grad_()
    loss = P.distill_loss(leaf, v, ids, tail, lengths, 2.0)
    loss.sum().backward()
    want, loss_tol, grad, tol = R.distill(small, *(a.cpu() for a in (v, ids, tail, lengths)), temperature=2.0)
    R.near(loss, want, loss_tol)
    R.near(leaf.grad, grad, R.rounded_bound(grad, tol, "bf16"))
    there = R.frames(lengths, B, T)
    p, q = (torch.softmax(a.cpu().double() / 2.0, -1) for a in (big, small))
    at = ids.cpu().long().clamp(min=0)
    coarse = [torch.cat([a.gather(2, at), 1 - a.gather(2, at).sum(-1, keepdim=True)], -1) for a in (p, q)]
    kl = (coarse[0] * (coarse[0] / coarse[1]).log()).sum(-1)
    assert ((loss.cpu().double() - kl)[there].abs() < 1e-4).all()


def operators(B, T, W, kind="bf16", k=12, seed=1):
    """Each operator as a call on buffers of its own, and what it writes."""
    d, g = dev(), gen(seed)
    x = scores(B, T, W, kind, seed)
    v, ids, tail = (a.to(d) for a in teacher(B, T, W, k, seed))
    h = torch.randint(0, W, (B, 50), generator=g, dtype=torch.int32).to(d)
    out = torch.zeros((B, T, W), device=d)
    tv, ti, tt = torch.zeros((B, T, k), device=d), torch.zeros((B, T, k), dtype=torch.int32, device=d), torch.zeros((B, T), device=d)
    loss, grad = torch.zeros((B, T), device=d), torch.zeros((B, T, W), dtype=x.dtype, device=d)
    return x, [
        (lambda **s: P.process_logits(x, history=h, repetition=1.2, presence=0.3, out=out, **s), [out]),
        (lambda **s: P.top_logits(x, k, values=tv, ids=ti, tail=tt, **s), [tv, ti, tt]),
        (lambda **s: P.distill(x, v, ids, tail, loss=loss, grad=grad, **s), [loss, grad]),
    ]


@pytest.mark.parametrize("B,T,W", [(2, 30, 1025), (2, 3, 9001), (1, 2, 140000)])
def test_streams(B, T, W):
    """On a stream of the caller's, as an object and as a handle, with torch's current stream another one."""
    x, ops = operators(B, T, W)
    torch.cuda.synchronize()
    for call, outs in ops:
        call()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        s = torch.cuda.Stream()
        for stream in (s, s.cuda_stream):
            for o in outs:
                o.zero_()
            torch.cuda.synchronize()
            call(stream=stream)
            s.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("B,T,W", [(2, 30, 1025), (2, 3, 9001), (1, 2, 140000)])
def test_graphs(B, T, W):
    """Two captured graphs, replayed in turn on new inputs with eager calls between."""
    x, ops = operators(B, T, W)
    for call, outs in ops:
        call()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for call, outs in ops:
                call()
        graphs.append(g)
    for i in range(4):
        x.copy_(scores(B, T, W, "bf16", 50 + i))
        for call, outs in ops:
            call()
        torch.cuda.synchronize()
        want = [o.clone() for _, outs in ops for o in outs]
        for _, outs in ops:
            for o in outs:
                o.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([o for _, outs in ops for o in outs], want)), f"replay {i}"


def test_top_tail_is_the_same_every_time():
    """Many labels above the bound, found by many waves in any order."""
    for W, k in ((9000, 128), (60000, 128), (60000, 64), (200000, 100)):
        x = scores(2, 3, W, "bf16", W)
        first = P.top_logits(x, k)
        for _ in range(20):
            assert all(torch.equal(a, b) for a, b in zip(P.top_logits(x, k), first))


def test_distill_loss_is_not_captured():
    x = scores(1, 2, 40, "fp32", 1).requires_grad_()
    v, ids, tail = (a.to(dev()) for a in teacher(1, 2, 40, 4, 1))
    P.distill_loss(x, v, ids, tail)
    torch.cuda.synchronize()
    y, g = torch.zeros(4, device=dev()), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y += 1
        with pytest.raises(RuntimeError, match="not captured"):
            P.distill_loss(x, v, ids, tail)
        loss = P.distill_loss(x.detach(), v, ids, tail)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(loss, P.distill_loss(x.detach(), v, ids, tail))


def test_same_call_same_bits():
    for B, T, W in ((3, 20, 1025), (2, 2, 20001), (1, 2, 200001), (130, 1, 20001)):
        x, ops = operators(B, T, W)
        for call, outs in ops:
            call()
            first = [o.clone() for o in outs]
            for _ in range(3):
                call()
                assert all(torch.equal(a, b) for a, b in zip(outs, first))


def test_offsets_beyond_32_bits():
    """A row that starts more than 2^32 bytes into its buffer."""
    W, d = 1025, dev()
    far = 2 ** 31 + 4096                              # elements of 2 bytes
    buf = torch.empty(far + W, dtype=torch.bfloat16, device=d)
    x = torch.as_strided(buf, (2, 1, W), (far, W, 1))
    fresh = scores(2, 1, W, "bf16", 9)
    x.copy_(fresh)
    v, ids, tail = (a.to(d) for a in teacher(2, 1, W, 8, 3))
    assert torch.equal(P.process_logits(x), P.process_logits(fresh))
    assert all(torch.equal(a, b) for a, b in zip(P.top_logits(x, 8), P.top_logits(fresh, 8)))
    grad = torch.as_strided(torch.empty(far + W, dtype=torch.bfloat16, device=d), (2, 1, W), (far, W, 1))
    a, b = P.distill(x, v, ids, tail, grad=grad), P.distill(fresh, v, ids, tail)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_refusals_of_device_tensors():
    d = dev()
    x = scores(2, 3, 40, "fp32", 1)
    v, ids, tail = (a.to(d) for a in teacher(2, 3, 40, 4, 1))
    for call, error in (
            (lambda: P.process_logits(x[0]), ValueError),
            (lambda: P.process_logits(x.double()), TypeError),
            (lambda: P.process_logits(x.transpose(1, 2)), ValueError),
            (lambda: P.process_logits(x, torch.zeros(3, dtype=torch.int32, device=d)), ValueError),
            (lambda: P.process_logits(x, torch.zeros(2, dtype=torch.int64, device=d)), TypeError),
            (lambda: P.process_logits(x, torch.zeros(2, dtype=torch.int32)), TypeError),
            (lambda: P.process_logits(x, mask=torch.zeros(2, 3, dtype=torch.int32, device=d)), ValueError),
            (lambda: P.process_logits(x, bias=torch.zeros(3, 40, device=d)), ValueError),
            (lambda: P.process_logits(x, penalties=torch.ones(2, 2, device=d)), ValueError),
            (lambda: P.process_logits(x, history=torch.zeros(3, 4, dtype=torch.int32, device=d)), ValueError),
            (lambda: P.process_logits(x, history=torch.zeros(2, 4, device=d)), TypeError),
            (lambda: P.process_logits(x, history_lengths=torch.zeros(2, dtype=torch.int32, device=d)), ValueError),
            (lambda: P.process_logits(x, repetition=0.0), P.CtcbeamError),
            (lambda: P.process_logits(x, out=x.transpose(0, 1)), ValueError),
            (lambda: P.process_logits(x.bfloat16(), out=x.bfloat16()), TypeError),
            (lambda: P.top_logits(x, 0), P.CtcbeamError),
            (lambda: P.top_logits(x, 41), P.CtcbeamError),
            (lambda: P.top_logits(x, 129), P.CtcbeamError),
            (lambda: P.top_logits(x, 4, temperature=0.0), P.CtcbeamError),
            (lambda: P.top_logits(x, 4, ids=torch.zeros(2, 3, 4, device=d)), TypeError),
            (lambda: P.distill(x, v[:, :2], ids), ValueError),
            (lambda: P.distill(x, v, None), TypeError),
            (lambda: P.distill(x, v, ids.long()), TypeError),
            (lambda: P.distill(x, v, ids, tail[:1]), ValueError),
            (lambda: P.distill(x, v, ids, weights=torch.ones(2, device=d)), ValueError),
            (lambda: P.distill(x, v, ids, grad=x), P.CtcbeamError),
            (lambda: P.distill(x, v, ids, grad=torch.empty(2, 3, 40, dtype=torch.float16, device=d)), TypeError),
            (lambda: P.distill(x, v, ids, want_loss=False, want_grad=False), P.CtcbeamError)):
        with pytest.raises(error):
            call()


def test_no_rows():
    d = dev()
    for B, T in ((0, 4), (3, 0)):
        x = torch.zeros(B, T, 17, device=d)
        v, ids = torch.zeros(B, T, 3, device=d), torch.zeros(B, T, 3, dtype=torch.int32, device=d)
        assert P.process_logits(x).shape == (B, T, 17)
        assert [tuple(a.shape) for a in P.top_logits(x, 3)] == [(B, T, 3), (B, T, 3), (B, T)]
        assert [tuple(a.shape) for a in P.distill(x, v, ids)] == [(B, T), (B, T, 17)]
