"""Arguments that the operators on rows of scores may not accept, at both sides
of their limits, through the C entry points on the CPU.  Calls that the limits
allow are stopped by a refusal that is checked later; no address is used."""
import struct

import pytest

import paper_2508_07315_amd as P
from test_rows_refusals import A, LONG, distill, process, rows, top


def message():
    return P._load().ctcbeam_last_error().decode()


def fp32(bits):
    return struct.unpack("f", struct.pack("I", bits))[0]


# 1/t is finite from 2.9387359e-39 on, log2(e)/t from 4.2396332e-39 on: in fp32
# bits, steps of 2^-149, 2097152 (whose quotient is 2^128) and 3025485
@pytest.mark.parametrize("temperature,good", [
    (fp32(2097153), False), (fp32(2500000), False), (fp32(3025400), False), (3e-39, False), (4.2e-39, False),
    (fp32(3025600), True), (4.3e-39, True), (1e-30, True), (1.0, True), (1e30, True), (3.4e38, True)])
def test_temperature(temperature, good):
    for call in (lambda: top(rows(), temperature=temperature, values=None), lambda: distill(rows(), temperature=temperature, values=None)):
        assert call() == 1
        assert ("null" if good else "temperature") in message()


# the longest row's arguments, each with its size in bytes; the row lies at A, its scores at 64 A
W = P.MAX_LABELS
INPUTS = dict(lengths=(8 * A, 4), history=(16 * A, 4 * 1000), history_lengths=(17 * A, 4), penalties=(18 * A, 12),
              bias=(20 * A, 4 * W), mask=(32 * A, W // 8))


@pytest.mark.parametrize("name", INPUTS)
def test_process_workspace_on_an_input(name):
    """The first launch would write where others, and the second one, still read."""
    lib = P._load()
    n = lib.ctcbeam_process_workspace_bytes(1, 1, W)
    given = {k: v[0] for k, v in INPUTS.items()}
    lengths = given.pop("lengths")
    at, size = INPUTS[name]
    for ws in (at, at + (size - 1) // 16 * 16, at - (n - 1) // 16 * 16):
        assert process(rows(**LONG, lengths=lengths), out=64 * A, history_size=1000, ws=ws, wn=n, **given) == 1
        assert message() == "workspace overlaps another argument"
