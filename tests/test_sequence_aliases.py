"""Outputs of the token-sequence calls that are inputs or each other are refused (no GPU: nothing is launched when validation fails)."""
import ctypes

import pytest

from paper_2601_22275_amd import binding
from tests.test_sequence_refusals import INT, INVALID, T, refuses

NAMES = ("q", "k", "v", "out", "d_out", "dq", "dk", "dv")


def backward(x, twin=""):
    fn = getattr(binding.lib(), "vmonarch_packed_attention_bwd" + twin)
    return fn(x["q"], x["k"], x["v"], x["out"], x["d_out"], INT, x["dq"], x["dk"], x["dv"], INT, INT, 1, 8, 8, 2, 2, 64, 1.0, 1, ctypes.c_void_p(256), 16, None)


@pytest.mark.parametrize("twin", ["", "_f32"])
@pytest.mark.parametrize("output", NAMES[5:])
def test_a_gradient_in_place_of_another_tensor(output, twin):
    """The same descriptor twice, and two descriptors of the same memory."""
    for other in NAMES:
        if other == output:
            continue
        x = {n: T((1 << 16) + (i << 12)) for i, n in enumerate(NAMES)}
        x[output] = x[other]
        refuses(INVALID, backward(x, twin), "must")
        x[output] = T((1 << 16) + (NAMES.index(other) << 12))
        refuses(INVALID, backward(x, twin), "must not be")
    x = {n: T((1 << 16) + (i << 12)) for i, n in enumerate(NAMES)}
    refuses(-3, backward(x, twin), "needed")  # eight tensors apart get as far as the workspace


def test_rotary_outputs_at_another_tensors_address():
    """An output may be its own input; where two of the four tensors are written by one launch, another's address is refused."""
    lib, plan = binding.lib(), ctypes.byref(binding.rotary_plan([16]))
    for twin in ("", "_f32"):
        def go(q, qo, k, ko, stride=8):
            return getattr(lib, "vmonarch_rotary" + twin)(T(q), T(qo), 4, T(k), T(ko), 4, 8, 64, INT, stride, plan, 0, None)

        a, b, c, e = (i << 16 for i in range(1, 5))
        for tensors in ((a, b, c, b), (a, c, c, e), (a, b, c, a), (a, a, a, a), (a, b, b, e)):
            refuses(INVALID, go(*tensors), "another tensor")
        for tensors in ((a, b, c, e), (a, a, c, c), (a, b, a, e)):  # apart, both in place, one input read twice
            refuses(INVALID, go(*tensors, stride=-1), "axis_stride")  # the next check
