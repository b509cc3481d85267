"""Sizes that do not fit the library's 32-bit ints are refused before anything
is allocated; their low bits alone would pass for a small, allowed size.

On the CPU: tensors of these sizes are stood in for by shapes without memory."""
import pytest
import torch

import paper_2508_07315_amd as P

FAR = 2 ** 32                                     # its low 32 bits are 0


class Shape(torch.Tensor):
    """A device tensor's shape, strides and type."""
    @staticmethod
    def __new__(cls, *shape, dtype=torch.float32):
        return torch.Tensor._make_wrapper_subclass(cls, shape, device="cuda:0", dtype=dtype)

    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise AssertionError(f"{func} before the refusal")

    def data_ptr(self):
        return 1 << 20


def refused(call, what):
    with pytest.raises(P.CtcbeamError, match=f"{what} = .* does not fit 32 bits") as e:
        call()
    assert e.value.code == 2


@pytest.mark.parametrize("what,shape", [("B", (FAR + 2, 3, 5)), ("T", (2, FAR + 3, 5)), ("W", (2, 3, FAR + 5)), ("W", (2, 3, 2 ** 31))])
def test_rows(what, shape):
    x = Shape(*shape, dtype=torch.bfloat16)
    v, i = Shape(*shape[:2], 2), Shape(*shape[:2], 2, dtype=torch.int32)
    for call in (lambda: P.process_logits(x), lambda: P.top_logits(x, 2), lambda: P.distill(x, v, i), lambda: P.distill_loss(x, v, i)):
        refused(call, what)


@pytest.mark.parametrize("n", [FAR + 7, 2 ** 31])
def test_histories_and_lists(n):
    x = Shape(2, 3, 5)
    refused(lambda: P.process_logits(x, out=Shape(2, 3, 5), history=Shape(2, n, dtype=torch.int32)), "history_size")
    refused(lambda: P.top_logits(x, n), "k")
    refused(lambda: P.distill(x, Shape(2, 3, n), Shape(2, 3, n, dtype=torch.int32)), "k")


@pytest.mark.parametrize("decode", [P.ctcbeam_decode, P.ctcbeam_decode_ex, P.ctcbeam_decode_nbest, P.ctcbeam_decode_noalloc])
def test_decoders(decode):
    n = Shape(2, dtype=torch.int32)
    for what, shape in (("B", (FAR + 2, 3, 5)), ("T", (2, FAR + 3, 5)), (r"V\+1", (2, 3, FAR + 5))):
        refused(lambda: decode(Shape(*shape), n, 4), what)
        refused(lambda: P.ctcbeam_greedy_decode(Shape(*shape), n), what)
    refused(lambda: decode(Shape(2, 3, 5), n, FAR + 4), "K")


def test_builders_and_workspace():
    refused(lambda: P.ctcbeam_boost_build_host(FAR + 9, [0, 1], [3]), "vocab_size")
    refused(lambda: P.ctcbeam_lm_build_arpa_host("none.arpa", FAR + 9), "vocab_size")
    refused(lambda: P.ctcbeam_workspace_bytes(2, FAR + 3, 4), "T")
    with pytest.raises(P.CtcbeamError):           # (what fits is the library's to check)
        P.ctcbeam_boost_build_host(-1, [0, 1], [3])
