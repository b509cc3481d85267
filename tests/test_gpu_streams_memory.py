"""The memory of tensors that a call allocates for a launch on another stream
than torch's current one."""
import pytest
import torch

import paper_2508_07315_amd as P
from test_gpu_rows import dev, scores, teacher

pytestmark = pytest.mark.gpu
B, T, W, K = 3, 50, 40, 4


def calls():
    """Calls that allocate their outputs, as functions of the stream, each with the tensors it makes."""
    x = P.process_logits(scores(B, T, W, "fp32", 1))
    long = scores(1, 2, 200000, "fp32", 2)
    n = torch.tensor([T, 7, 0], dtype=torch.int32, device=dev())
    v, i, t = (a.to(dev()) for a in teacher(B, T, W, K, 3))
    torch.cuda.synchronize()
    return [lambda s: P.ctcbeam_process_logits(x, stream=s), lambda s: P.ctcbeam_process_logits(long, stream=s),
            lambda s: P.ctcbeam_top_logits(x, K, stream=s), lambda s: P.ctcbeam_top_logits(long, K, stream=s),
            lambda s: P.ctcbeam_distill(x, v, i, t, stream=s), lambda s: P.ctcbeam_decode(x, n, K, stream=s),
            lambda s: P.ctcbeam_decode_nbest(x, n, K, stream=s), lambda s: P.ctcbeam_greedy_decode(x, n, stream=s),
            lambda s: P.ctcbeam_decode_noalloc(x, n, K, stream=s)]


def blocks(result):
    return {t.data_ptr(): t.numel() * t.element_size() for t in result if t is not None}


@pytest.mark.parametrize("handle", [False, True])
def test_memory_that_the_current_stream_freed_is_left_alone(handle):
    """Work queued on the current stream may still use it."""
    s = torch.cuda.Stream()
    for call in calls():
        want = call(None)
        torch.cuda.synchronize()
        freed = [torch.empty(n, dtype=torch.uint8, device=dev()) for n in blocks(want).values() for _ in range(4)]
        freed_at = {t.data_ptr() for t in freed}
        del freed
        got = call(s.cuda_stream if handle else s)
        torch.cuda.synchronize()
        assert not freed_at & set(blocks(got))
        outputs = [(a, b) for a, b in zip(got, want) if a is not None and a.dtype != torch.uint8]
        assert all(torch.equal(a, b) for a, b in outputs)


def test_outputs_in_use_on_the_current_stream_are_not_reused():
    """An output freed while the current stream still has work with it is not the next call's."""
    s = torch.cuda.Stream()
    for call in calls():
        got = call(s)
        s.synchronize()
        torch.cuda._sleep(20_000_000)
        at = set(blocks(got))
        del got
        again = call(s)
        reused = at & set(blocks(again))
        torch.cuda.synchronize()
        assert not reused
        del again


def test_the_default_stream_by_its_handle():
    """Handle 0, with the default stream current and with another one."""
    for call in calls():
        want = call(None)
        torch.cuda.synchronize()
        for current in (torch.cuda.default_stream(), torch.cuda.Stream()):
            with torch.cuda.stream(current):
                got = call(0)
            torch.cuda.synchronize()
            outputs = [(a, b) for a, b in zip(got, want) if a is not None and a.dtype != torch.uint8]
            assert all(torch.equal(a, b) for a, b in outputs)
