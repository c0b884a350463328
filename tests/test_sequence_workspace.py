"""Workspace of the backward pass: what a call needs, no more (no GPU: nothing is launched when the workspace is too small)."""
import ctypes

import pytest
import torch

from paper_2601_22275_amd import binding
from tests.test_sequence_refusals import INT, T

NAMES = ("q", "k", "v", "out", "d_out", "dq", "dk", "dv")
SIZES = [(3, 9000, 9000, 12, 4, 128), (1, 100000, 128, 4, 2, 64), (2, 700, 33, 5, 5, 200), (1, 1, 1, 1, 1, 1)]


def needed(twin, n, tq, tk, hq, hk, d, stride):
    """Bytes the call asks for, from its refusal of too few."""
    x = [T((1 << 16) + (i << 12), stride, stride) for i in range(len(NAMES))]
    fn = getattr(binding.lib(), "vmonarch_packed_attention_bwd" + twin)
    rc = fn(*x[:5], INT, *x[5:], INT, INT, n, tq, tk, hq, hk, d, 1.0, 1, ctypes.c_void_p(256), 1, None)
    text = binding.lib().vmonarch_last_error().decode()
    assert rc == -3 and "needed" in text, (rc, text)
    return int(text.split("bytes, ")[1].split()[0])


@pytest.mark.parametrize("n,tq,tk,hq,hk,d", SIZES)
def test_backward_workspace(n, tq, tk, hq, hk, d):
    """Two statistics a row, rounded up to 256 bytes; partial gradients of keys only where the bf16 matrix units run: bf16 on 16-byte rows, d <= 128."""
    lib = binding.lib()
    rows = -(-tq * hq * 8 // 256) * 256
    assert needed("_f32", n, tq, tk, hq, hk, d, 256) == rows
    assert lib.vmonarch_packed_attention_bwd_workspace_bytes_f32(n, tq, tk, hq, hk, d) == rows
    assert needed("", n, tq, tk, hq, hk, d, 257) == rows
    assert needed("", n, tq, tk, hq, hk, d, 256) <= lib.vmonarch_packed_attention_bwd_workspace_bytes(n, tq, tk, hq, hk, d)
    if d % 8 == 0:
        assert needed("", n, tq, tk, hq, hk, d, 256) == lib.vmonarch_packed_attention_bwd_workspace_bytes(n, tq, tk, hq, hk, d)


def test_sizes_that_are_none():
    for f in ("", "_f32"):
        size = getattr(binding.lib(), "vmonarch_packed_attention_bwd_workspace_bytes" + f)
        assert size(1, 0, 8, 4, 2, 64) == 0 and size(1, 8, 8, 4, 3, 64) == 0 and size(0, 8, 8, 4, 2, 64) == 0 and size(1, 8, 8, 4, 2, 257) == 0


@pytest.mark.gpu
def test_the_binding_allocates_what_the_twin_needs():
    n, heads, kv, d = 3000, 4, 2, 64
    q, do = (torch.randn(n, heads, d, device="cuda") for _ in range(2))
    k, v = (torch.randn(n, kv, d, device="cuda") for _ in range(2))
    s = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out, lse = binding.packed_attention(q, k, v, s, lse=True)
    grads = [torch.empty_like(x) for x in (q, k, v)]
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    binding.packed_attention_bwd(q, k, v, out, do, lse, s, dq=grads[0], dk=grads[1], dv=grads[2])
    assert torch.cuda.max_memory_allocated() - before <= -(-n * heads * 8 // 512) * 512  # (torch's allocator deals in 512 bytes)
