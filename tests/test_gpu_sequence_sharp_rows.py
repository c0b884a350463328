"""Gradients of rows whose weight sits on a few keys, on the GPU."""
import math

import numpy as np
import pytest
import torch

from tests import sequence_oracle as S
from tests.test_gpu_sequences import B, f64, starts, tokens  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


def rounded_once(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("d,group,order", [(64, 1, "token"), (128, 2, "token"), (136, 1, "token"), (64, 2, "odd")])
@pytest.mark.parametrize("nk", [400, 600, 4000])
@pytest.mark.parametrize("deviation,offset", [(2, 0.0), (8, 0.0), (16, 0.0), (2, 3.0)])
def test_gradients_of_sharp_rows(B, d, group, order, nk, deviation, offset):  # noqa: F811
    """Errors in the 2-norm against those of the exact gradient rounded once.  dS and P are rounded once as matrix operands, the result once more: two
    independent roundings of the same relative size, the root of two in place of one; the limit is two.  offset: what all keys have in common, which a
    row's gradient does not depend on."""
    gen = torch.Generator().manual_seed(d + nk + deviation)
    nq = 150
    q, do = tokens(gen, nq, group, d, "bf16", order, deviation), tokens(gen, nq, group, d, "bf16", order)
    k, v = tokens(gen, nk, 1, d, "bf16", order), tokens(gen, nk, 1, d, "bf16", order)
    k += offset
    qs, ks = starts([nq]), starts([nk])
    out, lse = B.packed_attention(q, k, v, qs, ks, causal=False, lse=True)
    grads = B.packed_attention_bwd(q, k, v, out, do, lse, qs, ks, causal=False)
    want = S.packed(f64(q), f64(k), f64(v), [0, nq], [0, nk], float(np.float32(1.0 / math.sqrt(d))), False, "bf16", f64(do))
    ratios = {}
    for name, g in zip(("dq", "dk", "dv"), grads):
        ref = want[name][0]
        ratios[name] = np.linalg.norm(f64(g) - ref) / np.linalg.norm(rounded_once(ref) - ref)
    print("  error in roundings:", {n: round(r, 3) for n, r in ratios.items()})
    assert max(ratios.values()) < 2.0, ratios
