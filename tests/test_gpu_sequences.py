"""Token-sequence operators on the GPU against their 64-bit forms, element by element within derived bounds."""
import math

import numpy as np
import pytest
import torch

from tests import sequence_oracle as S

pytestmark = pytest.mark.gpu
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def B():
    from paper_2601_22275_amd import binding
    binding.lib()
    return binding


def starts(lengths, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lengths)]), dtype=torch.int32, device="cuda")


def tokens(gen, n, heads, d, dtype, order="token", scale=1.0):
    shape = {"token": (n, heads, d), "head": (heads, n, d), "fused": (n, 3 * heads, d), "odd": (n, heads, d + 1)}[order]
    x = (torch.randn(shape, generator=gen) * scale).to(TYPE[dtype]).cuda()
    if order == "head":
        return x.transpose(0, 1)
    if order == "fused":
        return x[:, heads:2 * heads]
    if order == "odd":
        return x[..., :d]
    return x


def f64(x):
    return x.detach().double().cpu().numpy()


def within(name, got, want):
    ref, bound = want
    g = f64(got)
    rows = ~np.isnan(ref)
    with np.errstate(invalid="ignore", over="ignore"):
        bad = rows & ~((np.abs(g - ref) <= bound) | (g == ref))
        ratio = np.nanmax(np.where(rows & np.isfinite(ref), np.abs(g - ref) / np.maximum(bound, 1e-30), 0.0), initial=0.0)
    print(f"  {name}: largest error / bound {ratio:.3f}")
    assert not bad.any(), (name, np.argwhere(bad)[:5], g[bad][:5], ref[bad][:5])


CASES = [
    # dtype, d, kv heads, group, query lengths, key lengths (None: the same), causal, order
    ("bf16", 64, 2, 3, [1, 5, 130, 64, 65], None, True, "token"),
    ("bf16", 64, 4, 1, [300, 1, 257], None, False, "head"),
    ("bf16", 128, 1, 4, [33, 0, 400, 31], None, True, "token"),
    ("bf16", 128, 3, 1, [129, 600], None, True, "fused"),
    ("bf16", 128, 2, 2, [7, 150], [500, 33], True, "token"),       # the second has rows that see nothing
    ("bf16", 128, 2, 1, [70, 40, 3], [0, 77, 513], False, "head"),  # ... and the first of these no keys at all
    ("bf16", 64, 1, 8, [1, 1, 1], [1, 64, 1000], True, "token"),
    ("bf16", 96, 2, 2, [100, 50], None, True, "token"),
    ("bf16", 80, 1, 5, [90], [210], False, "fused"),
    ("bf16", 8, 2, 1, [40, 90], None, True, "token"),
    ("bf16", 72, 2, 1, [40, 90], None, True, "head"),
    ("bf16", 100, 2, 1, [40, 41], None, True, "token"),
    ("bf16", 64, 2, 2, [70, 33], None, True, "odd"),
    ("bf16", 200, 1, 2, [65, 20], None, True, "token"),
    ("bf16", 256, 1, 1, [40], [100], False, "token"),
    ("f32", 64, 2, 2, [1, 100, 64], None, True, "token"),
    ("f32", 128, 1, 3, [50, 0, 90], [50, 20, 10], True, "head"),
    ("f32", 32, 3, 1, [65, 127], None, False, "fused"),
    ("f32", 1, 1, 2, [9], None, True, "token"),
    ("f32", 33, 2, 1, [40, 30], None, True, "odd"),
    ("f32", 256, 1, 2, [37], [80], False, "token"),
]


@pytest.mark.parametrize("dtype,d,kv,group,ql,kl,causal,order", CASES)
def test_packed_attention_and_its_gradients(B, dtype, d, kv, group, ql, kl, causal, order):
    gen = torch.Generator().manual_seed(len(ql) * 1000 + d + group)
    kl = ql if kl is None else kl
    q = tokens(gen, sum(ql), kv * group, d, dtype, order, 1.5)
    k = tokens(gen, sum(kl), kv, d, dtype, order, 1.3)
    v = tokens(gen, sum(kl), kv, d, dtype, order)
    do = tokens(gen, sum(ql), kv * group, d, dtype, order)
    qs, ks = starts(ql), starts(kl)
    out, lse = B.packed_attention(q, k, v, qs, ks, causal=causal, lse=True)
    assert torch.equal(out, B.packed_attention(q, k, v, qs, ks, causal=causal))  # with and without the log-sum-exp, twice the same bits
    scale = float(np.float32(1.0 / math.sqrt(d)))
    want = S.packed(f64(q), f64(k), f64(v), qs.tolist(), ks.tolist(), scale, causal, dtype, f64(do))
    within("out", out, want["out"])
    within("lse", lse, want["lse"])
    grads = B.packed_attention_bwd(q, k, v, out, do, lse, qs, ks, causal=causal)
    for name, g in zip(("dq", "dk", "dv"), grads):
        within(name, g, want[name])
    again = B.packed_attention_bwd(q, k, v, out, do, lse, qs, ks, causal=causal)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("dtype,d,n,causal", [("bf16", 128, 2300, True), ("bf16", 64, 2111, False), ("bf16", 64, 1800, True), ("bf16", 128, 1111, False)])
def test_long_rows_with_growing_maxima(B, dtype, d, n, causal):
    """Row maxima that jump from tile to tile, by more than float's exponent range too: later keys are larger.  Few rows are compared."""
    gen = torch.Generator().manual_seed(n)
    q, k, v = (tokens(gen, n, 2, d, dtype, "token", s) for s in (1.0, 1.0, 1.0))
    grow = torch.ones(n)
    grow[::97] = 8.0
    grow[n // 2:: 211] = 60.0
    k = (k.float() * grow.cuda()[:, None, None]).to(TYPE[dtype])
    s = starts([n])
    out, lse = B.packed_attention(q, k, v, s, causal=causal, lse=True)
    rows = np.unique(np.concatenate([np.arange(0, n, 97), [n - 1, n // 2, n // 2 + 1]]))
    scale = float(np.float32(1.0 / math.sqrt(d)))
    for h in range(2):
        for i in rows:
            m = i + 1 if causal else n
            r = S.attention(f64(q[i:i + 1, h]), f64(k[:m, h]), f64(v[:m, h]), scale, False, dtype)
            for name, got in (("out", out[i, h]), ("lse", lse[h, i])):
                ref, bound = r[name]
                assert (np.abs(f64(got) - ref[0]) <= bound[0]).all(), (name, h, i, f64(got), ref[0], bound[0])


def test_rows_of_no_sequence_are_neither_read_nor_written(B):
    for dtype in ("bf16", "f32"):
        gen = torch.Generator().manual_seed(5)
        n, first, lens = 200, 7, [60, 0, 70]
        q, k, v, do = (tokens(gen, n, h, 64, dtype) for h in (4, 2, 2, 4))
        s = starts(lens, first)
        inside = slice(first, first + sum(lens))
        for x in (q, k, v, do):
            x[:first] = math.nan
            x[first + sum(lens):] = math.nan
        out = torch.full_like(q, 3.0)
        out, lse = B.packed_attention(q, k, v, s, lse=True, out=out)
        grads = [torch.full_like(x, 3.0) for x in (q, k, v)]
        B.packed_attention_bwd(q, k, v, out, do, lse, s, dq=grads[0], dk=grads[1], dv=grads[2])
        for x in [out] + grads:
            assert torch.isfinite(x[inside]).all()
            assert (x[:first] == 3).all() and (x[first + sum(lens):] == 3).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_what_a_row_does_not_see_does_not_reach_it(B, dtype, d):
    gen = torch.Generator().manual_seed(6)
    n, bad = 190, 100
    q, k, v = (tokens(gen, 2 * n, h, d, dtype) for h in (2, 1, 1))
    s = starts([n, n])
    # Not bit for bit the same: where values are not finite keys are added one at a time, nk fp32 additions in another order
    # (nk 2^-24 of the weighted magnitudes, which the bound has).
    want = S.packed(f64(q), f64(k), f64(v), [0, n, 2 * n], [0, n, 2 * n], float(np.float32(1.0 / math.sqrt(d))), True, dtype)["out"]
    want[0][bad:n] = math.nan  # rows that see the key are looked at below
    for kv_value, v_value in ((math.nan, math.nan), (0.0, math.inf), (math.inf, 0.0)):
        k2, v2 = k.clone(), v.clone()
        k2[bad], v2[bad] = k2[bad] + kv_value, v2[bad] + v_value
        out = B.packed_attention(q, k2, v2, s)
        within("out", out, want)
        assert not torch.isfinite(out[bad:n]).all(-1).any() or kv_value == math.inf
    # logits of -inf alone: zeros and a log-sum-exp of -inf
    q2, k2 = q.abs() + 0.5, k.clone()
    k2[:bad] = -math.inf
    out, lse = B.packed_attention(q2, k2, v, s, lse=True)
    assert (out[:bad] == 0).all() and torch.isneginf(lse[:, :bad]).all() and torch.isfinite(out[bad:]).all() and torch.isfinite(lse[:, bad:]).all()


def test_broadcast_inputs_and_slices(B):
    gen = torch.Generator().manual_seed(7)
    q = tokens(gen, 90, 4, 64, "bf16", "fused")
    k1 = tokens(gen, 90, 1, 64, "bf16")
    k = k1.expand(90, 4, 64)  # one head shown as four: head stride 0
    s = starts([40, 50])
    assert torch.equal(B.packed_attention(q, k, k, s), B.packed_attention(q, k.contiguous(), k.contiguous(), s))
    assert torch.equal(B.packed_attention(q, k, k, s), B.packed_attention(q, k1, k1, s))


def test_starts_out_of_range_stay_in_bounds(B):
    gen = torch.Generator().manual_seed(8)
    q, k, v = (tokens(gen, 50, 2, 64, "bf16") for _ in range(3))
    s = torch.tensor([-5, 20, 1000], dtype=torch.int32, device="cuda")
    out = B.packed_attention(q, k, v, s)
    assert torch.equal(out, B.packed_attention(q, k, v, starts([20, 30])))


# ---- rotary -------------------------------------------------------------------------------------------------------------------

ROTARY = [
    # dtype, d, heads, kv heads, axis pairs, interleaved, kwargs of the plan, first position, order
    ("bf16", 128, 3, 3, [22, 21, 21], True, {}, 0, "head"),
    ("bf16", 128, 4, 1, [64], False, {}, 1_000_000, "token"),
    ("bf16", 64, 5, 2, [16], False, dict(factor=4.0), 0, "fused"),
    ("bf16", 64, 1, 1, [13], True, dict(factor=8.0, context=512.0, low_turns=1.0, high_turns=32.0, amplitude=1.3), 77, "token"),
    ("bf16", 80, 2, 1, [5, 4, 4], False, {}, 0, "odd"),
    ("f32", 96, 5, 1, [32], False, dict(factor=8.0, context=8192.0, low_turns=1.0, high_turns=32.0, amplitude=1.2), 2 ** 30, "token"),
    ("f32", 33, 2, 2, [16], True, {}, -3, "token"),
    ("f32", 256, 1, 1, [128], False, dict(base=500.0), 5, "head"),
    ("f32", 2, 9, 3, [1], True, {}, 123456789, "token"),
]


@pytest.mark.parametrize("n", [1, 37, 700])
@pytest.mark.parametrize("dtype,d,heads,kv,pairs,inter,kw,first,order", ROTARY)
def test_rotary(B, dtype, d, heads, kv, pairs, inter, kw, first, order, n):
    gen = torch.Generator().manual_seed(n + d)
    q, k = tokens(gen, n, heads, d, dtype, order), tokens(gen, n, kv, d, dtype, order)
    pos = torch.stack([first + torch.arange(n) % (50 + 10 * a) if a else first + torch.arange(n) for a in range(len(pairs))]).to(torch.int32)
    plan = B.rotary_plan(pairs, interleaved=inter, **kw)
    f = S.frequencies(pairs, kw.get("base", 1e4), kw.get("factor", 1.0), kw.get("context", 0.0), kw.get("low_turns", 0.0), kw.get("high_turns", 0.0))
    amplitude = kw.get("amplitude", 1.0)
    for backward in (False, True):
        got = B.rotary(q, k, pos.cuda(), plan, backward=backward)
        for x, y in zip((q, k), got):
            want = S.rotary(f64(x), pos.numpy(), pairs, f, inter, backward, amplitude)
            # positions beyond 2^26 make the oracle's own angle (64-bit products of up to 2^30 with frequencies rounded once) off by 2^-23
            within("turned", y, (want, S.rotary_bound(f64(x), want, pairs, inter, amplitude, dtype)))
            rest = 2 * sum(pairs)
            assert torch.equal(x[..., rest:], y[..., rest:])
    alone, none = B.rotary(q, None, pos.cuda(), plan)
    assert none is None and torch.equal(alone, B.rotary(q, k, pos.cuda(), plan)[0])
    q2, k2 = q.clone(), k.clone()
    B.rotary(q2, k2, pos.cuda(), plan, q_out=q2, k_out=k2)  # in place
    for a, b in zip((q2, k2), B.rotary(q, k, pos.cuda(), plan)):
        assert torch.equal(a, b)


# ---- pages --------------------------------------------------------------------------------------------------------------------


def pages(gen, lengths, page, kv, d, dtype, order="page"):
    """A cache with room for the lengths, of NaN, its pages dealt at random, and the table."""
    per = [-(-n // page) for n in lengths]
    n = sum(per) + 2
    shape = {"page": (n, page, kv, d), "head": (n, kv, page, d), "odd": (n, page, kv, d + 1)}[order]
    made = []
    for _ in range(2):
        x = torch.full(shape, math.nan, dtype=TYPE[dtype], device="cuda")
        made.append(x.transpose(1, 2) if order == "head" else x[..., :d] if order == "odd" else x)
    order_ = torch.randperm(n, generator=gen)
    table = torch.full((len(lengths), max(max(per), 1) + 1), -7, dtype=torch.int32)
    at = 0
    for s, p in enumerate(per):
        table[s, :p] = order_[at:at + p].to(torch.int32)
        at += p
    return made[0], made[1], table.cuda()


PAGED = [
    # dtype, d, kv, group, chunk lengths, cached lengths, page, causal, order
    ("bf16", 64, 2, 3, [1, 1, 1, 1], [1, 17, 300, 64], 16, True, "page"),
    ("bf16", 128, 1, 8, [1, 1], [2000, 37], 64, True, "page"),
    ("bf16", 128, 2, 5, [1, 0, 1], [129, 40, 513], 7, True, "head"),
    ("bf16", 128, 3, 1, [40, 1, 0, 200], [500, 1, 30, 200], 39, False, "page"),
    ("bf16", 64, 2, 2, [33, 70], [1030, 70], 1, True, "page"),
    ("bf16", 96, 2, 2, [1, 20], [300, 33], 16, True, "page"),
    ("bf16", 64, 1, 40, [1, 3], [400, 100], 16, True, "page"),
    ("bf16", 128, 1, 1, [1], [9000], 128, True, "page"),
    ("bf16", 64, 2, 2, [1, 9], [100, 200], 16, True, "odd"),
    ("bf16", 200, 1, 2, [1, 9], [100, 200], 16, False, "page"),
    ("f32", 64, 2, 2, [1, 30], [500, 90], 16, True, "page"),
    ("f32", 40, 1, 3, [5], [5], 3, False, "head"),
]


@pytest.mark.parametrize("dtype,d,kv,group,new,have,page,causal,order", PAGED)
def test_append_then_paged_attention(B, dtype, d, kv, group, new, have, page, causal, order):
    """A cache written in two goes (everything before the chunks, then the chunks) and read by the chunks."""
    gen = torch.Generator().manual_seed(page + d)
    ck, cv, table = pages(gen, have, page, kv, d, dtype, order)
    old = [b - a for a, b in zip(new, have)]
    k, v = tokens(gen, sum(have), kv, d, dtype, "token", 1.3), tokens(gen, sum(have), kv, d, dtype)
    q = tokens(gen, sum(new), kv * group, d, dtype, "fused", 1.5)
    ends = np.cumsum(have)
    is_old = np.concatenate([np.r_[np.ones(o, bool), np.zeros(n, bool)] for o, n in zip(old, new)])
    int32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    if sum(old):
        at = torch.from_numpy(np.flatnonzero(is_old)).cuda()
        B.paged_append(k[at], v[at], ck, cv, table, starts(old), int32(old))
    at = torch.from_numpy(np.flatnonzero(~is_old)).cuda()
    B.paged_append(k[at], v[at], ck, cv, table, starts(new), int32(have))
    assert int(torch.isfinite(ck.float()).all(-1).all(-1).sum()) == sum(have)  # these slots and no other
    got = B.paged_attention(q, ck, cv, table, starts(new), int32(have), causal=causal)
    want = S.packed(f64(q), f64(k), f64(v), np.r_[0, np.cumsum(new)], np.r_[0, ends], float(np.float32(1.0 / math.sqrt(d))), causal, dtype)
    within("out", got, want["out"])
    assert torch.equal(got, B.paged_attention(q, ck, cv, table, starts(new), int32(have), causal=causal))


def test_lengths_and_pages_out_of_range(B):
    gen = torch.Generator().manual_seed(9)
    for dtype in ("bf16", "f32"):
        ck, cv, table = pages(gen, [64, 64], 16, 2, 64, dtype)
        ck.zero_(), cv.zero_()
        table = table[:, :4].contiguous()
        k, v, q = (tokens(gen, 10, h, 64, dtype) for h in (2, 2, 4))
        before = ck.clone()
        table[0] = torch.tensor([-1, 99, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
        s = starts([5, 5])
        long = torch.tensor([64, 2 ** 31 - 1], dtype=torch.int32, device="cuda")  # the second is cut to the table's 64
        B.paged_append(k, v, ck, cv, table, s, long)
        changed = (ck != before).any(-1).any(-1)
        assert int(changed.sum()) == 5 and changed[int(table[1, 3]), 11:].all()  # the bad pages' tokens went nowhere
        out = B.paged_attention(q, ck, cv, table, s, long)
        assert torch.equal(out[5:], B.paged_attention(q, ck, cv, table, s, torch.tensor([64, 64], dtype=torch.int32, device="cuda"))[5:])
        short = torch.tensor([-3, 2], dtype=torch.int32, device="cuda")  # chunks longer than what is there: rows that see nothing
        out = B.paged_attention(q, ck, cv, table, s, short)
        assert (out[:8] == 0).all()
        before = ck.clone()
        B.paged_append(k, v, ck, cv, table, s, short)  # tokens at positions below zero go nowhere
        assert int((ck != before).any(-1).any(-1).sum()) <= 2


def test_a_cache_beyond_32_bits(B):
    """Pages past 2^32 bytes and 2^31 elements of the cache."""
    d, kv, page = 128, 8, 256
    n = 2 ** 31 // (d * kv * page) + 9
    ck, cv = (torch.empty((n, page, kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gen = torch.Generator().manual_seed(10)
    have = 3 * page - 5
    table = torch.tensor([[n - 1, 2, n - 3]], dtype=torch.int32, device="cuda")
    k, v = tokens(gen, have, kv, d, "bf16"), tokens(gen, have, kv, d, "bf16")
    q = tokens(gen, have, 2 * kv, d, "bf16")
    length = torch.tensor([have], dtype=torch.int32, device="cuda")
    B.paged_append(k, v, ck, cv, table, starts([have]), length)
    assert torch.equal(ck[n - 3, :page - 5], k[2 * page:]) and torch.equal(cv[n - 1], v[:page])
    want = S.packed(f64(q[-2:]), f64(k), f64(v), [0, 2], [0, have], float(np.float32(1.0 / math.sqrt(d))), True, "bf16")
    within("out", B.paged_attention(q[-2:].contiguous(), ck, cv, table, starts([2]), length), want["out"])
    got = B.paged_attention(q, ck, cv, table, starts([have]), length)
    within("out", got[-2:], want["out"])


# ---- together -----------------------------------------------------------------------------------------------------------------


def test_a_layer_token_by_token_and_at_once(B):
    """Rotary positions, cache and attention, chunk after chunk (a frame, a few tokens, single ones), against the whole sequence at once."""
    gen = torch.Generator().manual_seed(11)
    d, kv, heads, page, lens = 128, 2, 6, 10, [75, 130]
    q, k, v = (tokens(gen, sum(lens), h, d, "bf16") for h in (heads, kv, kv))
    plan = B.rotary_plan([48], interleaved=True, factor=2.0)
    pos = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
    tq, tk = B.rotary(q, k, pos, plan)
    whole = B.packed_attention(tq, tk, v, starts(lens))
    ck, cv, table = pages(gen, lens, page, kv, d, "bf16")
    out = torch.full_like(whole, math.nan)
    done = [0, 0]
    for chunk in ([39, 39], [30, 0], [0, 60], [5, 7], [1, 1], [0, 1], [0, 20], [0, 2]):
        at = torch.cat([sum(lens[:s]) + done[s] + torch.arange(c) for s, c in enumerate(chunk)]).cuda()
        done = [a + c for a, c in zip(done, chunk)]
        have, s = torch.tensor(done, dtype=torch.int32, device="cuda"), starts(chunk)
        B.paged_append(k[at], v[at], ck, cv, table, s, have, plan=plan)  # at the tokens' positions in their sequence
        out[at] = B.paged_attention(B.rotary(q[at], None, pos[at], plan)[0], ck, cv, table, s, have)
    assert done == lens
    want = S.packed(f64(tq), f64(tk), f64(v), np.r_[0, np.cumsum(lens)], np.r_[0, np.cumsum(lens)], float(np.float32(1.0 / math.sqrt(d))), True, "bf16")
    within("whole", whole, want["out"])
    within("chunks", out, want["out"])


def test_captured_calls_replay_on_new_data(B):
    """Two graphs of the same calls, replayed in turn with eager work between, each against the eager result."""
    gen = torch.Generator().manual_seed(12)
    d, kv, heads, lens = 64, 2, 4, [50, 90, 700]
    s, n = starts(lens), sum(lens)
    plan = B.rotary_plan([32])
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    one, have = starts([1, 1, 1]), torch.tensor(lens, dtype=torch.int32, device="cuda")
    ck, cv, table = pages(gen, lens, 16, kv, d, "bf16")

    def step(q, k, v, do):
        tq, tk = B.rotary(q, k, pos, plan)
        out, lse = B.packed_attention(tq, tk, v, s, lse=True)
        grads = B.packed_attention_bwd(tq, tk, v, out, do, lse, s)
        B.paged_append(tk, v, ck, cv, table, s, have)
        return (out, lse) + grads + (B.paged_attention(q[:3], ck, cv, table, one, have),)

    def inputs():
        return [tokens(gen, n, h, d, "bf16") for h in (heads, kv, kv, heads)]

    graphs = []
    for _ in range(2):
        x = inputs()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(*x)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y = step(*x)
        graphs.append((g, x, y))
    for _ in range(3):
        for g, x, y in graphs:
            for a, b in zip(x, inputs()):
                a.copy_(b)
            g.replay()
            got = [t.clone() for t in y]
            torch.cuda.synchronize()
            for a, b in zip(got, step(*x)):
                assert torch.equal(a, b)


def test_calls_on_another_stream(B):
    gen = torch.Generator().manual_seed(13)
    q, k, v = (tokens(gen, 300, 2, 128, "bf16") for _ in range(3))
    s = starts([100, 200])
    want = B.packed_attention(q, k, v, s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = B.packed_attention(q, k, v, s)
    side.synchronize()
    assert torch.equal(got, want)


def test_binding_refusals(B):
    x = torch.zeros((8, 4, 64), dtype=torch.bfloat16, device="cuda")
    s = starts([8])
    bad = [
        lambda: B.packed_attention(x, x[:, :3], x[:, :3], s),                               # 4 heads on 3
        lambda: B.packed_attention(x, x.float(), x.float(), s),                             # types
        lambda: B.packed_attention(x, x, x[:4], s),                                         # shapes of k and v
        lambda: B.packed_attention(x, x, x, s.long()),                                      # int64 starts
        lambda: B.packed_attention(x, x, x, s, starts([4, 4])),                             # two counts of sequences
        lambda: B.packed_attention(x[0], x[0], x[0], s),                                    # two dimensions
        lambda: B.packed_attention(x.half(), x.half(), x.half(), s),                        # fp16
        lambda: B.packed_attention(x[..., ::2], x[..., ::2], x[..., ::2], s),               # channels apart
        lambda: B.packed_attention(x, x, x, s, out=x),                                      # in place
        lambda: B.packed_attention(x, x, x, s, scale=0.0),
        lambda: B.packed_attention_bwd(x, x, x, x.clone(), x, torch.zeros(4, 9, device="cuda"), s),  # lse of another call
        lambda: B.rotary(x, None, torch.zeros(7, dtype=torch.int32, device="cuda"), B.rotary_plan([32])),
        lambda: B.rotary(x, x[:4], torch.zeros(8, dtype=torch.int32, device="cuda"), B.rotary_plan([32])),
        lambda: B.rotary(x, None, torch.zeros(8, dtype=torch.int32, device="cuda"), B.rotary_plan([33])),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(B.VMonarchError):
            f()
            print("accepted:", i)


@pytest.mark.parametrize("d,kv,group,n,causal", [(64, 12, 1, 5700, True), (64, 6, 2, 5700, False), (128, 12, 1, 5700, True), (64, 2, 1, 2100, False)])
def test_launches_of_many_workgroups(B, d, kv, group, n, causal):
    """More workgroups than run at once (other tiles at d = 64), keys packed and in pages; a few rows of every head are compared."""
    gen = torch.Generator().manual_seed(n + d)
    lens = [n, n // 3 + 1]
    heads = kv * group
    q, k, v = tokens(gen, sum(lens), heads, d, "bf16", "token", 1.5), tokens(gen, sum(lens), kv, d, "bf16", "token", 1.3), tokens(gen, sum(lens), kv, d, "bf16")
    s, have = starts(lens), torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = B.packed_attention(q, k, v, s, causal=causal, lse=True)
    assert torch.equal(out, B.packed_attention(q, k, v, s, causal=causal))
    ck, cv, table = pages(gen, lens, 100, kv, d, "bf16")
    B.paged_append(k, v, ck, cv, table, s, have)
    paged = B.paged_attention(q, ck, cv, table, s, have, causal=causal)
    scale = float(np.float32(1.0 / math.sqrt(d)))
    kc, vc = f64(k), f64(v)
    for a, m in zip((0, n), lens):
        rows = np.unique([0, 31, 127, 128, m // 2, m - 1])
        for h in range(heads):
            g = h // group
            for i in rows:
                seen = i + 1 if causal else m
                r = S.attention(f64(q[a + i:a + i + 1, h]), kc[a:a + seen, g], vc[a:a + seen, g], scale, False, "bf16")
                for name, got in (("out", out[a + i, h]), ("out", paged[a + i, h]), ("lse", lse[h, a + i])):
                    ref, bound = r[name]
                    assert (np.abs(f64(got) - ref[0]) <= bound[0]).all(), (name, h, i)


@pytest.mark.parametrize("dtype,d,page", [("bf16", 64, 16), ("bf16", 128, 7), ("bf16", 33, 4), ("f32", 64, 16)])
@pytest.mark.parametrize("causal", [True, False])
def test_more_sequences_than_a_wave_has_lanes(B, dtype, d, page, causal):
    """150 sequences, some empty on one side, short and of a few tiles; every element, forward, backward and over pages."""
    rng = np.random.default_rng(d)
    ql, kl = rng.integers(0, 6, 150), rng.integers(0, 9, 150)
    ql[[3, 70, 149]], kl[[3, 70, 149]] = [90, 40, 130], [90, 77, 20]
    gen = torch.Generator().manual_seed(d)
    q, do = (tokens(gen, int(ql.sum()), 4, d, dtype) for _ in range(2))
    k, v = (tokens(gen, int(kl.sum()), 2, d, dtype) for _ in range(2))
    qs, ks = starts(ql), starts(kl)
    out, lse = B.packed_attention(q, k, v, qs, ks, causal=causal, lse=True)
    want = S.packed(f64(q), f64(k), f64(v), qs.tolist(), ks.tolist(), float(np.float32(1.0 / math.sqrt(d))), causal, dtype, f64(do))
    within("out", out, want["out"])
    within("lse", lse, want["lse"])
    for name, g in zip(("dq", "dk", "dv"), B.packed_attention_bwd(q, k, v, out, do, lse, qs, ks, causal=causal)):
        within(name, g, want[name])
    ck, cv, table = pages(gen, kl, page, 2, d, dtype)
    have = torch.tensor(kl, dtype=torch.int32, device="cuda")
    B.paged_append(k, v, ck, cv, table, ks, have)
    within("paged", B.paged_attention(q, ck, cv, table, qs, have, causal=causal), want["out"])


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_large_values_do_not_overflow(B, dtype, d):
    """Values around 2^95 and logits that grow along the row."""
    gen = torch.Generator().manual_seed(21)
    n = 900
    q, k, v = (tokens(gen, n, 2, d, dtype, "token", s) for s in (1.0, 2.0, 2.0 ** 95))
    k = (k.float() * torch.linspace(0.2, 3.0, n, device="cuda")[:, None, None]).to(TYPE[dtype])
    s = starts([n])
    want = S.packed(f64(q), f64(k), f64(v), [0, n], [0, n], float(np.float32(1.0 / math.sqrt(d))), True, dtype)
    within("out", B.packed_attention(q, k, v, s), want["out"])
    ck, cv, table = pages(gen, [n], 16, 2, d, dtype)
    have = torch.tensor([n], dtype=torch.int32, device="cuda")
    B.paged_append(k, v, ck, cv, table, s, have)
    within("paged", B.paged_attention(q[-3:], ck, cv, table, starts([3]), have), (want["out"][0][-3:], want["out"][1][-3:]))
    within("paged", B.paged_attention(q[-300:], ck, cv, table, starts([300]), have), (want["out"][0][-300:], want["out"][1][-300:]))


@pytest.mark.parametrize("d,kv,group,ql,kl,causal", [(64, 2, 2, [1500, 700], [200, 130], False), (128, 1, 2, [1300], None, True), (72, 1, 4, [700, 0, 900], [40, 10, 333], True)])
def test_gradients_of_keys_that_many_rows_see(B, d, kv, group, ql, kl, causal):
    """Few keys under many rows: the rows are cut into ranges whose sums meet in memory.  The first two tokens and the last belong to no sequence."""
    gen = torch.Generator().manual_seed(d)
    kl = ql if kl is None else kl
    assert B.lib().vmonarch_packed_attention_bwd_workspace_bytes(len(ql), sum(ql), sum(kl), kv * group, kv, d) > 16 * sum(ql) * kv * group  # ranges
    q, do = (tokens(gen, sum(ql) + 3, kv * group, d, "bf16", "head") for _ in range(2))
    k, v = (tokens(gen, sum(kl) + 3, kv, d, "bf16", "fused") for _ in range(2))
    qs, ks = starts(ql, 2), starts(kl, 2)
    out, lse = B.packed_attention(q, k, v, qs, ks, causal=causal, lse=True)
    dk, dv = torch.full_like(k, 3.0), torch.full_like(v, 3.0)
    dq, dk, dv = B.packed_attention_bwd(q, k, v, out, do, lse, qs, ks, causal=causal, dk=dk, dv=dv)
    want = S.packed(f64(q), f64(k), f64(v), qs.tolist(), ks.tolist(), float(np.float32(1.0 / math.sqrt(d))), causal, "bf16", f64(do))
    for name, g in (("dq", dq), ("dk", dk), ("dv", dv)):
        within(name, g[2:-1], tuple(x[2:-1] for x in want[name]))
    for x in (dk, dv):
        assert (x[:2] == 3).all() and (x[-1] == 3).all()


CHUNKS = [
    # many rows over caches long enough to be cut into ranges of keys; the last two: whole prompts
    ("bf16", 128, 2, 1, [150, 1, 60], [3000, 900, 2100], 64, True, "page"),
    ("bf16", 128, 1, 3, [129], [2600], 390, False, "head"),
    ("bf16", 72, 2, 2, [90, 0, 40], [1500, 0, 1800], 39, True, "page"),
    ("bf16", 64, 1, 1, [128], [2049], 3, True, "page"),
    ("f32", 64, 1, 2, [60, 100], [1500, 100], 16, True, "page"),
    ("bf16", 200, 1, 1, [70], [1300], 16, False, "page"),
    ("bf16", 128, 2, 2, [700], [700], 16, True, "page"),
    ("bf16", 64, 2, 1, [300, 512, 77], [300, 512, 77], 32, True, "page"),
]


@pytest.mark.parametrize("dtype,d,kv,group,new,have,page,causal,order", CHUNKS)
def test_chunks_over_long_caches(B, dtype, d, kv, group, new, have, page, causal, order):
    test_append_then_paged_attention(B, dtype, d, kv, group, new, have, page, causal, order)
