"""Rows whose logits are finite and large, on the GPU."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_sequences import B, f64, pages, starts, tokens  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu


def one_hot_logits(n, heads, kv, d, dtype, size, nq):
    """Logits -size * (1 + j / 64) for key j at scale 1: every row's weight sits on its first key, and the logits are exact."""
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    root = 2.0 ** (round(math.log2(size)) // 2)
    q, k = torch.zeros(nq, heads, d), torch.zeros(n, kv, d)
    q[..., 0] = -root
    k[..., 0] = size / root * (1 + torch.arange(n)[:, None] / 64)
    return q.to(kind).cuda(), k.to(kind).cuda()


@pytest.mark.parametrize("dtype,size", [("bf16", 2.0 ** 20), ("bf16", 2.0 ** 28), ("f32", 2.0 ** 28), ("f32", 2.0 ** 102)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sign", [-1, 1])
def test_rows_of_large_logits(B, dtype, size, d, sign):  # noqa: F811
    """Finite logits of any size that fp32 has (bf16 matrix units: up to 2^28) leave a row its result: packed, over pages, and over pages in ranges of
    keys.  The one key with the largest logit is the row's result to the last bit; the log-sum-exp is that logit, through two products with
    constants in fp32 (2^-22 of it)."""
    n, nq, heads, kv = 60, 40, 2, 1
    gen = torch.Generator().manual_seed(d)
    q, k = one_hot_logits(n, heads, kv, d, dtype, size, nq)
    if sign > 0:
        q, k = -q, k.flip(0).contiguous()
    logit = f64(q)[0, 0, 0] * f64(k)[0, 0, 0]
    best = 0
    v = tokens(gen, n, kv, d, dtype)
    out, lse = B.packed_attention(q, k, v, starts([nq]), starts([n]), causal=False, scale=1.0, lse=True)
    assert (out == v[best]).all()
    assert (np.abs(f64(lse) - logit) <= 2.0 ** -22 * abs(logit)).all()
    ck, cv, table = pages(gen, [n], 16, kv, d, dtype)
    have = torch.tensor([n], dtype=torch.int32, device="cuda")
    B.paged_append(k, v, ck, cv, table, starts([n]), have)
    for rows in (1, nq):  # the kernel for few rows, the one for many
        for wide in (4, 1024):  # pages a row of the table has room for: uncut, in ranges
            t = torch.zeros((1, wide), dtype=torch.int32, device="cuda")
            t[:, :4] = table[:, :4]
            paged = B.paged_attention(q[:rows], ck, cv, t, starts([rows]), have, causal=False, scale=1.0)
            assert (paged == v[best]).all(), (rows, wide)
