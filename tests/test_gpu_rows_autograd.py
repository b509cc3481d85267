"""Outputs that a caller gives are written where torch sees it: a backward pass
that saved one of them before fails, and does not read what is there now."""
import pytest
import torch

import paper_2508_07315_amd as P
from test_gpu_rows import dev, scores, teacher

pytestmark = pytest.mark.gpu
CHANGED = "modified by an inplace operation"


def lists(seed, B=2, T=3, W=40, k=4):
    v, i, t = (a.to(dev()) for a in teacher(B, T, W, k, seed))
    return v, i, t


@pytest.mark.parametrize("again", ["values", "ids", "tail"])
def test_a_list_written_again_before_backward(again):
    """One teacher's list reused for the next while the first loss still waits for its backward pass."""
    v, i, t = lists(1)
    student = scores(2, 3, 40, "fp32", 2).requires_grad_()
    loss = P.distill_loss(student, v, i, t)
    new = dict(zip(("values", "ids", "tail"), lists(3)))
    new[again] = dict(values=v, ids=i, tail=t)[again]
    P.top_logits(scores(2, 3, 40, "fp32", 4), 4, **new)
    with pytest.raises(RuntimeError, match=CHANGED):
        loss.sum().backward()


def test_a_student_processed_in_place_before_backward():
    student = scores(2, 3, 40, "fp32", 2).requires_grad_()
    loss = P.distill_loss(student, *lists(1))
    P.process_logits(student.detach(), out=student.detach())
    with pytest.raises(RuntimeError, match=CHANGED):
        loss.sum().backward()


def test_loss_and_gradient_buffers_written_again():
    v, i, t = lists(1)
    student = scores(2, 3, 40, "fp32", 2)
    a = torch.ones(2, 3, device=dev(), requires_grad=True)
    b = torch.ones(2, 3, 40, device=dev(), requires_grad=True)
    loss, grad = torch.zeros(2, 3, device=dev()), torch.zeros(2, 3, 40, device=dev())
    for leaf, given in ((a, dict(loss=loss, want_grad=False)), (b, dict(grad=grad[:, :, :], want_loss=False))):
        y = (leaf * (loss if leaf is a else grad)).sum()
        P.distill(student, v, i, t, **given)
        with pytest.raises(RuntimeError, match=CHANGED):
            y.backward()


def test_decoded_scores_written_again():
    lp = P.process_logits(scores(2, 9, 12, "fp32", 5))
    n = torch.tensor([9, 4], dtype=torch.int32, device=dev())
    _, _, sc, _ = P.ctcbeam_decode(lp, n, 4)
    leaf = torch.ones(2, device=dev(), requires_grad=True)
    y = (leaf * sc).sum()
    P.ctcbeam_decode(lp, n, 4, out_scores=sc)
    with pytest.raises(RuntimeError, match=CHANGED):
        y.backward()


def test_untouched_lists_still_differentiate():
    """New outputs, and outputs under no_grad or of inference mode, are no error."""
    v, i, t = lists(1)
    student = scores(2, 3, 40, "fp32", 2).requires_grad_()
    loss = P.distill_loss(student, v, i, t)
    P.top_logits(scores(2, 3, 40, "fp32", 4), 4)
    P.process_logits(student.detach())
    loss.sum().backward()
    assert torch.equal(student.grad, P.distill(student.detach(), v, i, t)[1])
    with torch.no_grad():
        P.process_logits(student, out=student)
    with torch.inference_mode():
        out = torch.zeros(2, 3, 40, device=dev())
        P.process_logits(student.detach(), out=out)
    P.process_logits(student.detach(), out=out)


def test_outputs_that_require_a_gradient_are_refused():
    x = scores(2, 3, 40, "fp32", 2).requires_grad_()
    lists_ = lists(1)
    f = lambda *shape: torch.zeros(*shape, device=dev(), requires_grad=True)  # noqa: E731
    for call in (lambda: P.process_logits(x, out=x), lambda: P.process_logits(x * 2, out=x * 2),
                 lambda: P.top_logits(x, 4, values=f(2, 3, 4)), lambda: P.top_logits(x, 4, tail=f(2, 3)),
                 lambda: P.distill(x, *lists_, loss=f(2, 3)), lambda: P.distill(x, *lists_, grad=f(2, 3, 40))):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
