"""Every key of a sequence is read once, and by the rows that see it: queries of zero give all keys a row sees the same weight, and values that are
one in a single channel name the key.  A key read twice or not at all is a factor of two or zero in that channel."""
import ctypes
import math

import pytest
import torch

from tests.test_gpu_sequences import B, TYPE, pages, starts, tokens  # noqa: F401 (B is a fixture)

pytestmark = pytest.mark.gpu

# A weight is one and its sum a whole number, both exact; what is left is the quotient's rounding to the stored type (half a step: 2^-8 or 2^-24 of it)
# and, in fp32, the quotient and the ranges' log-sums (a logarithm of up to 2^4 and its exponential: 2^-19).
TOLERANCE = {"bf16": 2.0 ** -8 + 2.0 ** -18, "f32": 2.0 ** -18}


def names(n, heads, d, dtype, first):
    """[n, heads, d]: key first + head * d + channel has a one there."""
    x = torch.zeros((n, heads, d), dtype=TYPE[dtype], device="cuda")
    i = torch.arange(heads * d, device="cuda")
    i = i[first + i < n]
    x[first + i, i // d, i % d] = 1
    return x


def seen(nq, nk, causal):
    """Keys a row sees, and which: [nq, nk]"""
    i, j = torch.arange(nq, device="cuda")[:, None], torch.arange(nk, device="cuda")[None]
    return j <= nk - nq + i if causal else (j >= 0).expand(nq, nk)


def expected(nq, nk, heads, d, first, causal):
    sees = seen(nq, nk, causal).double()
    weight = sees / sees.sum(1, keepdim=True).clamp(min=1.0)
    n = heads * d
    w = torch.zeros((nq, max(first + n, nk)), dtype=torch.float64, device="cuda")
    w[:, :nk] = weight
    return w[:, first:first + n].reshape(nq, heads, d)


def check(got, want, dtype, what):
    bad = (got.double() - want).abs() > TOLERANCE[dtype] * want
    assert not bad.any(), (what, bad.nonzero()[:5].tolist(), got[bad][:5].tolist(), want[bad][:5].tolist())


PACKED = [
    # dtype, d, kv heads, group, query lengths, key lengths, causal
    ("bf16", 128, 2, 1, [1, 130, 40], [700, 257, 33], True),
    ("bf16", 128, 2, 2, [200], [1089], False),
    ("bf16", 64, 2, 3, [90, 31], [545, 64], True),
    ("bf16", 64, 4, 1, [1000], [1000], True),
    ("bf16", 64, 12, 1, [1500, 1300], [1500, 1300], True),  # more workgroups than run at once: tiles of 32 keys
    ("bf16", 72, 2, 1, [100], [417], False),
    ("bf16", 136, 1, 1, [70], [300], True),
    ("f32", 64, 2, 1, [70, 3], [129, 95], True),
    ("f32", 256, 1, 1, [40], [161], False),
]


@pytest.mark.parametrize("dtype,d,kv,group,ql,kl,causal", PACKED)
def test_packed_keys(B, dtype, d, kv, group, ql, kl, causal):  # noqa: F811
    q = torch.zeros((sum(ql), kv * group, d), dtype=TYPE[dtype], device="cuda")
    gen = torch.Generator().manual_seed(d)
    k = tokens(gen, sum(kl), kv, d, dtype)
    for first in range(0, max(kl), kv * d):
        v = torch.cat([names(n, kv, d, dtype, first) for n in kl])
        out = B.packed_attention(q, k, v, starts(ql), starts(kl), causal=causal)
        a = 0
        for s, (nq, nk) in enumerate(zip(ql, kl)):
            want = expected(nq, nk, kv, d, first, causal)
            for g in range(group):
                check(out[a:a + nq, g::group], want, dtype, (s, g, first))
            a += nq


PAGED = [
    # dtype, d, kv, group, chunk lengths, lengths, page, pages a row of the table has room for, causal, ranges
    ("bf16", 128, 2, 1, [1, 1], [700, 65], 16, 45, True, None),
    ("bf16", 128, 4, 5, [1], [2049], 16, 1024, True, 64),      # most ranges have no keys
    ("bf16", 128, 4, 1, [1, 1, 1], [9000, 1, 640], 128, 71, True, None),
    ("bf16", 64, 4, 3, [1, 2], [1500, 4097], 64, 512, True, 64),
    ("bf16", 64, 2, 2, [1] * 60, [300 + 7 * i for i in range(60)], 16, 45, False, None),
    ("bf16", 128, 4, 1, [150, 60], [2600, 2111], 7, 400, True, None),
    ("bf16", 128, 12, 1, [390, 380], [8190, 4000], 390, 21, False, None),
    ("bf16", 128, 12, 1, [2000] * 6, [2000, 1999, 1985, 1984, 33, 0], 64, 512, True, 5),
    ("bf16", 128, 12, 1, [1200] * 3, [2944, 2001, 1300], 64, 46, True, 2),
    ("bf16", 64, 12, 1, [300, 200], [3000, 3001], 16, 1024, False, None),
    ("bf16", 64, 4, 1, [512, 77], [512, 77], 32, 16, True, None),
    ("bf16", 136, 2, 1, [1, 40], [600, 513], 16, 100, True, None),
    ("f32", 64, 4, 2, [1, 33], [1500, 700], 16, 512, True, None),
    ("f32", 128, 2, 1, [1], [1025], 64, 17, True, None),
]


def ranges_of(B, c, n, tokens_, heads, kv, d):  # noqa: F811
    """Ranges of keys by the workspace that the call asks for (mask or none)."""
    size = B.lib().vmonarch_paged_attention_workspace_bytes(ctypes.byref(c), n, tokens_, heads, kv, d)
    padded = 64 if d <= 64 else 128 if d <= 128 else 256
    return max(1, size // (tokens_ * heads * (padded + 1) * 4))


@pytest.mark.parametrize("dtype,d,kv,group,new,have,page,width,causal,ranges", PAGED)
def test_paged_keys(B, dtype, d, kv, group, new, have, page, width, causal, ranges):  # noqa: F811
    """Caches whose other slots hold NaN, and tables as wide as the sequences or many times wider."""
    gen = torch.Generator().manual_seed(page + d)
    ck, cv, tight = pages(gen, have, page, kv, d, dtype)
    table = torch.full((len(have), width), -1, dtype=torch.int32, device="cuda")
    n = min(width, tight.shape[1])
    table[:, :n] = tight[:, :n]
    lengths = torch.tensor(have, dtype=torch.int32, device="cuda")
    if ranges is not None:
        c = B.Cache(n_pages=1, page_size=page, table_width=width)
        assert ranges_of(B, c, len(new), sum(new), kv * group, kv, d) == ranges
    q = torch.zeros((sum(new), kv * group, d), dtype=TYPE[dtype], device="cuda")
    k = tokens(gen, sum(have), kv, d, dtype)
    for first in range(0, max(have), kv * d):
        v = torch.cat([names(m, kv, d, dtype, first) for m in have])
        B.paged_append(k, v, ck, cv, table, starts(have), lengths)
        out = B.paged_attention(q, ck, cv, table, starts(new), lengths, causal=causal)
        a = 0
        for s, (nq, nk) in enumerate(zip(new, have)):
            want = expected(nq, nk, kv, d, first, causal)
            for g in range(group):
                check(out[a:a + nq, g::group], want, dtype, (s, g, first))
            a += nq


GRADIENTS = [
    # dtype, d, kv heads, group, query lengths, key lengths, causal
    ("bf16", 128, 2, 1, [150, 40], [257, 33], True),
    ("bf16", 128, 1, 2, [1300], [130], False),        # rows of queries in ranges
    ("bf16", 64, 2, 2, [1500, 700], [200, 130], False),
    ("bf16", 64, 4, 1, [700], [700], True),
    ("bf16", 128, 2, 1, [600], [1100], True),
    ("bf16", 136, 1, 1, [70], [300], True),
    ("f32", 64, 2, 1, [70, 3], [129, 95], True),
]


@pytest.mark.parametrize("dtype,d,kv,group,ql,kl,causal", GRADIENTS)
def test_gradients_of_every_pair(B, dtype, d, kv, group, ql, kl, causal):  # noqa: F811
    """P is 1 / (keys the row sees).  dv: d_out names the row.  dk: with k = 0 q names the row, dq: with q = 0 k names the key; there dP = +-1 by the key, so that
    dS = P (+-1 - their mean over the row's keys).  Roundings: P or dS as operands and the result, half a step each; dq: half a step more, should what the operands lose add up over
    the row."""
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    heads = kv * group
    nq, nk = sum(ql), sum(kl)
    gen = torch.Generator().manual_seed(nq + nk)
    kind = TYPE[dtype]
    qs, ks = starts(ql), starts(kl)
    sign = torch.where(torch.rand(nk, generator=gen) < 0.5, -1.0, 1.0).cuda()
    v = torch.zeros((nk, kv, d), dtype=kind, device="cuda")
    v[..., 0] = sign[:, None].to(kind)
    e0 = torch.zeros((nq, heads, d), dtype=kind, device="cuda")
    e0[..., 0] = 1
    zero_q, zero_k = torch.zeros((nq, heads, d), dtype=kind, device="cuda"), torch.zeros((nk, kv, d), dtype=kind, device="cuda")

    def grads(q, k, d_out):
        out, lse = B.packed_attention(q, k, v, qs, ks, causal=causal, scale=1.0, lse=True)
        return B.packed_attention_bwd(q, k, v, out, d_out, lse, qs, ks, causal=causal, scale=1.0)

    weights, signs = [], torch.split(sign.double(), kl)
    for a, b in zip(ql, kl):
        sees = seen(a, b, causal).double()
        weights.append(sees / sees.sum(1, keepdim=True).clamp(min=1.0))
    mean = [w @ s for w, s in zip(weights, signs)]
    for first in range(0, max(ql), d):
        x = torch.cat([names(n, 1, d, dtype, first) for n in ql]).expand(nq, heads, d)
        _, _, dv = grads(zero_q, tokens(gen, nk, kv, d, dtype), x)
        _, dk, _ = grads(x, zero_k, e0)
        at = 0
        for w, m, s, a, b in zip(weights, mean, signs, ql, kl):
            rows = slice(first, min(first + d, a))
            n = max(rows.stop - rows.start, 0)
            want = torch.zeros((b, d), dtype=torch.float64, device="cuda")
            size = torch.zeros_like(want)
            want[:, :n] = w[rows].T * group
            # (each head of the group adds a weight rounded alike)
            assert ((dv[at:at + b].double() - want[:, None]).abs() <= (2 * half + 2.0 ** -16) * want[:, None]).all(), first
            want[:, :n] = (w[rows] * (s[None] - m[rows, None])).T * group
            size[:, :n] = w[rows].T * 2 * group  # |+-1| + |mean|
            assert ((dk[at:at + b].double() - want[:, None]).abs() <= (2 * half + 2.0 ** -16) * size[:, None]).all(), first
            at += b
    for first in range(0, max(kl), d):
        x = torch.cat([names(n, 1, d, dtype, first) for n in kl]).expand(nk, kv, d)
        dq, _, _ = grads(zero_q, x, e0)
        at = 0
        for w, m, s, a, b in zip(weights, mean, signs, ql, kl):
            cols = slice(first, min(first + d, b))
            n = max(cols.stop - cols.start, 0)
            want, size = torch.zeros((a, d), dtype=torch.float64, device="cuda"), torch.zeros((a, d), dtype=torch.float64, device="cuda")
            want[:, :n] = w[:, cols] * (s[None, cols] - m[:, None])
            size[:, :n] = w[:, cols] * 2
            assert ((dq[at:at + a].double() - want[:, None]).abs() <= (3 * half + 2.0 ** -16) * size[:, None]).all(), first
            at += a


def test_a_table_cut_to_the_longest_sequence(B):  # noqa: F811
    """Rows of a wide table, shown as wide as the sequences need: the calls of a table of just that width, ranges included, to the last bit."""
    gen = torch.Generator().manual_seed(3)
    have, new, page, kv, heads, d = [700, 65, 512], [1, 40, 3], 16, 2, 4, 128
    ck, cv, tight = pages(gen, have, page, kv, d, "bf16")
    need = -(-max(have) // page)
    tight = tight[:, :need].contiguous()
    wide = torch.full((len(have), 4096), -1, dtype=torch.int32, device="cuda")
    wide[:, :need] = tight
    lengths = torch.tensor(have, dtype=torch.int32, device="cuda")
    B.paged_append(tokens(gen, sum(have), kv, d, "bf16"), tokens(gen, sum(have), kv, d, "bf16"), ck, cv, wide[:, :need], starts(have), lengths)
    q = tokens(gen, sum(new), heads, d, "bf16")
    for causal in (True, False):
        out = B.paged_attention(q, ck, cv, wide[:, :need], starts(new), lengths, causal=causal)
        assert torch.equal(out, B.paged_attention(q, ck, cv, tight, starts(new), lengths, causal=causal)) and torch.isfinite(out).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("bf16", 136), ("f32", 64)])
def test_no_keys_and_no_queries_at_all(B, dtype, d):  # noqa: F811
    """A batch without a single key: rows of zeros, log-sum-exps of -inf, gradients of zero.  Without a single query: the keys' gradients are zero."""
    gen = torch.Generator().manual_seed(d)
    some, none = starts([30, 0, 140]), starts([0, 0, 0])
    x = {h: tokens(gen, 170, h, d, dtype) for h in (4, 2)}
    y = {h: tokens(gen, 0, h, d, dtype) for h in (4, 2)}
    for causal in (True, False):
        out, lse = B.packed_attention(x[4], y[2], y[2], some, none, causal=causal, lse=True)
        assert (out == 0).all() and torch.isneginf(lse).all()
        dq, dk, dv = B.packed_attention_bwd(x[4], y[2], y[2], out, x[4], lse, some, none, causal=causal)
        assert (dq == 0).all() and dk.shape == dv.shape == (0, 2, d)
        out, lse = B.packed_attention(y[4], x[2], x[2], none, some, causal=causal, lse=True)
        dq, dk, dv = B.packed_attention_bwd(y[4], x[2], x[2], out, y[4], lse, none, some, causal=causal)
        assert dq.shape == (0, 4, d) and (dk == 0).all() and (dv == 0).all()
