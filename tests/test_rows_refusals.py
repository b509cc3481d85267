"""What the operators on rows of scores refuse, through the C entry points on
the CPU.  Only refused or empty calls are made, so the addresses are never
used."""
import ctypes

import pytest

import paper_2508_07315_amd as P

A = 1 << 20          # addresses far enough apart for the sizes below


def rows(data=A, type=0, B=2, T=3, W=10, sb=30, st=10, lengths=None):
    return P._Rows(data, type, B, T, W, sb, st, lengths)


def process(r, out=8 * A, ws=None, wn=0, **o):
    opts = P._ProcessOpts(**{"repetition": 1.0, "normalize": 1, **o})
    lib = P._load()
    return lib.ctcbeam_process_logits(None if r is None else ctypes.byref(r), ctypes.byref(opts), out, ws, wn, None)


def top(r, k=2, temperature=1.0, values=8 * A, ids=16 * A, tail=24 * A, ws=None, wn=0):
    lib = P._load()
    return lib.ctcbeam_top_logits(None if r is None else ctypes.byref(r), k, temperature, values, ids, tail, ws, wn, None)


def distill(r, k=2, temperature=1.0, values=8 * A, ids=16 * A, tail=24 * A, weights=None, weight=1.0, wsb=0, wst=0,
            loss=32 * A, grad=40 * A, gsb=30, gst=10, ws=None, wn=0):
    lib = P._load()
    return lib.ctcbeam_distill(None if r is None else ctypes.byref(r), values, ids, tail, k, temperature, weights, wsb, wst,
                               weight, loss, grad, gsb, gst, ws, wn, None)


CALLS = {"process": process, "top": top, "distill": distill}


@pytest.mark.parametrize("op", CALLS)
@pytest.mark.parametrize("code,message,change", [
    (1, "type", dict(type=3)),
    (1, "type", dict(type=-1)),
    (1, "B and T", dict(B=-1)),
    (1, "B and T", dict(T=-1)),
    (1, "W must", dict(W=0)),
    (2, "MAX_LABELS", dict(W=P.MAX_LABELS + 1)),
    (2, "MAX_ROWS", dict(B=1 << 10, T=(1 << 11) + 1)),
    (2, "MAX_ROWS", dict(B=(1 << 31) - 1, T=(1 << 31) - 1)),
    (1, "strides", dict(sb=-1)),
    (1, "strides", dict(st=-10)),
    (1, "null device", dict(data=None)),
    (1, "aligned", dict(data=A + 2)),
    (1, "aligned", dict(data=A + 1, type=2)),
    (1, "aligned", dict(lengths=A + 2)),
    (2, "strides too large", dict(sb=(1 << 63) - 1)),
])
def test_rows(op, code, message, change):
    assert CALLS[op](rows(**change)) == code
    assert message in P._load().ctcbeam_last_error().decode()


@pytest.mark.parametrize("op", CALLS)
def test_null_rows(op):
    assert CALLS[op](None) == 1


@pytest.mark.parametrize("op", CALLS)
@pytest.mark.parametrize("change", [dict(B=0), dict(T=0), dict(B=0, T=0, data=None)])
def test_no_rows_is_no_work(op, change):
    assert CALLS[op](rows(**change)) == 0


@pytest.mark.parametrize("code,message,change", [
    (1, "repetition", dict(repetition=0.0)),
    (1, "repetition", dict(repetition=-1.0)),
    (1, "repetition", dict(repetition=float("nan"))),
    (1, "repetition", dict(repetition=float("inf"))),
    (1, "presence", dict(presence=float("nan"))),
    (1, "presence", dict(frequency=float("inf"))),
    (1, "history_size", dict(history_size=-1)),
    (2, "history_size above", dict(history=2 * A, history_size=(1 << 30) + 1)),
    (2, "history_size above", dict(history=2 * A, history_size=(1 << 31) - 1)),
    (1, "null history", dict(history_size=4)),
    (1, "strides", dict(history=A, history_size=4, history_stride=-4)),
    (1, "strides", dict(bias=A, bias_stride=-10)),
    (1, "strides", dict(mask=A, mask_stride_b=-1)),
    (1, "strides", dict(mask=A, mask_stride_t=-1)),
    (2, "strides too large", dict(bias=2 * A, bias_stride=(1 << 63) - 1)),
    (1, "aligned", dict(bias=2 * A + 2)),
    (1, "aligned", dict(mask=2 * A + 1)),
    (1, "aligned", dict(penalties=2 * A + 1)),
    (1, "aligned", dict(history=2 * A + 1, history_size=3)),
    (1, "null output", dict(out=None)),
    (1, "aligned", dict(out=8 * A + 2)),
    (1, "overlaps an input", dict(bias=8 * A + 4)),
    (1, "overlaps an input", dict(mask=8 * A)),
    (1, "overlaps an input", dict(history=8 * A + 236, history_size=3)),
    (1, "overlaps an input", dict(penalties=8 * A - 8)),
])
def test_process(code, message, change):
    assert process(rows(), **change) == code
    assert message in P._load().ctcbeam_last_error().decode()


@pytest.mark.parametrize("change", [
    dict(data=8 * A + 4),                        # shifted by a label
    dict(data=8 * A, sb=40),                     # same place, other strides
    dict(data=8 * A, st=0, sb=0),
    dict(data=8 * A, type=2),                    # another type
])
def test_process_in_place_needs_the_same_rows(change):
    assert process(rows(**change)) == 1
    assert "overlaps the logits" in P._load().ctcbeam_last_error().decode()


@pytest.mark.parametrize("code,message,change", [
    (1, "k must", dict(k=0)),
    (1, "k must", dict(k=-3)),
    (2, "MAX_TOP", dict(k=P.MAX_TOP + 1)),
    (1, "k above W", dict(k=11)),
    (1, "temperature", dict(temperature=0.0)),
    (1, "temperature", dict(temperature=-1.0)),
    (1, "temperature", dict(temperature=float("nan"))),
    (1, "temperature", dict(temperature=float("inf"))),
    (1, "temperature", dict(temperature=1e-45)),
    (1, "null output", dict(values=None)),
    (1, "null output", dict(ids=None)),
    (1, "null output", dict(tail=None)),
    (1, "aligned", dict(values=8 * A + 2)),
    (1, "overlaps", dict(ids=8 * A + 44)),
    (1, "overlaps", dict(tail=16 * A + 4)),
    (1, "overlaps", dict(values=A)),
    (1, "overlaps", dict(tail=A + 236)),
])
def test_top(code, message, change):
    assert top(rows(), **change) == code
    assert message in P._load().ctcbeam_last_error().decode()


@pytest.mark.parametrize("code,message,change", [
    (1, "k must", dict(k=0)),
    (2, "MAX_TOP", dict(k=P.MAX_TOP + 1)),
    (1, "temperature", dict(temperature=0.0)),
    (1, "temperature", dict(temperature=float("nan"))),
    (1, "weight", dict(weight=float("nan"))),
    (1, "weight", dict(weight=float("inf"))),
    (1, "strides", dict(weights=2 * A, wsb=-1)),
    (1, "strides", dict(gst=-10)),
    (1, "null device", dict(values=None)),
    (1, "null device", dict(ids=None)),
    (1, "neither", dict(loss=None, grad=None)),
    (1, "aligned", dict(grad=40 * A + 2)),
    (1, "rows of grad", dict(gst=9)),
    (1, "rows of grad", dict(gsb=29)),
    (1, "rows of grad", dict(gsb=0)),
    (1, "rows of grad", dict(gst=0)),
    (1, "rows of grad", dict(gst=20, gsb=19)),
    (1, "overlaps", dict(grad=A)),
    (1, "overlaps", dict(grad=A + 236)),
    (1, "overlaps", dict(loss=40 * A + 4)),
    (1, "overlaps", dict(loss=8 * A)),
    (1, "overlaps", dict(grad=24 * A)),
    (1, "overlaps", dict(weights=40 * A + 8)),
])
def test_distill(code, message, change):
    assert distill(rows(), **change) == code
    assert message in P._load().ctcbeam_last_error().decode()


def test_python_wants_device_tensors():
    import torch
    x = torch.zeros(2, 3, 10)
    v, i = torch.zeros(2, 3, 2), torch.zeros(2, 3, 2, dtype=torch.int32)
    for call in (lambda: P.process_logits(x), lambda: P.top_logits(x, 2), lambda: P.distill(x, v, i),
                 lambda: P.distill_loss(x, v, i), lambda: P.process_logits([1.0])):
        with pytest.raises(TypeError, match="device tensor"):
            call()
    with pytest.raises(ValueError, match="constant"):
        P.distill_loss(x, v.requires_grad_(), i)


# a row of the most labels, which every operator cuts into spans: they need a workspace
LONG = dict(B=1, T=1, W=P.MAX_LABELS, sb=P.MAX_LABELS, st=P.MAX_LABELS)


@pytest.mark.parametrize("op,need,far", [
    ("process", lambda lib: lib.ctcbeam_process_workspace_bytes(1, 1, P.MAX_LABELS), dict(out=64 * A)),
    ("top", lambda lib: lib.ctcbeam_top_workspace_bytes(1, 1, P.MAX_LABELS, 2), {}),
    ("distill", lambda lib: lib.ctcbeam_distill_workspace_bytes(1, 1, P.MAX_LABELS), dict(grad=64 * A, gsb=P.MAX_LABELS, gst=P.MAX_LABELS)),
])
def test_workspace(op, need, far):
    lib = P._load()
    n = need(lib)
    assert n > 0
    for ws, wn, message in ((None, 0, "too small"), (None, n, "too small"), (48 * A, n - 1, "too small"),
                            (48 * A + 8, n, "aligned to 16"), (A + 64, n, "overlaps"), (64 * A if op != "top" else 8 * A, n, "overlaps")):
        assert CALLS[op](rows(**LONG), ws=ws, wn=wn, **far) == 1
        assert message in lib.ctcbeam_last_error().decode()


def test_workspace_of_nothing():
    lib = P._load()
    for B, T, W in ((0, 4, 100000), (4, 0, 100000), (-1, 4, 9), (4, 4, 0), (1, 1, P.MAX_LABELS + 1), (1 << 16, 1 << 16, 100000)):
        assert lib.ctcbeam_process_workspace_bytes(B, T, W) == 0
        assert lib.ctcbeam_top_workspace_bytes(B, T, W, 4) == 0
        assert lib.ctcbeam_distill_workspace_bytes(B, T, W) == 0
    assert lib.ctcbeam_top_workspace_bytes(1, 1, 262144, 0) == 0
    assert lib.ctcbeam_top_workspace_bytes(1, 1, 262144, 129) == 0
