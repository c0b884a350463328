"""What a video transformer's layers do with token sequences around Monarch attention, and what their speed is judged on:

  rotary   rotary positions of q and k (one to three position axes, interleaved or half layout, part of the head, scaled for long
           contexts), forward and backward                                                   binding.rotary
  append   new keys (rotated on the way) and values into a paged cache                       binding.paged_append
  paged    attention of each sequence's chunk of new tokens, or single token, over its pages  binding.paged_attention
  packed   attention over packed sequences of different lengths, causal or not, with grouped heads
                                                                                             binding.packed_attention
  train    the same with its log-sum-exp, then its backward pass                             binding.packed_attention_bwd

A case is a dict of plain values; `op` is one of the above.  Token tensors are [tokens, heads, d] views, stored token by token or
(order "head") head by head; heads = kv_heads * group.  Without `own` the operators are computed in plain torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

_GOLDEN = 0.6180339887498949


def _types(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _bytes(case):
    return 2 if case["dtype"] == "bf16" else 4


def _lengths(n, longest, shortest=1):
    """n lengths spread between `shortest` and `longest`, the first the longest; a function of the sizes alone."""
    return [longest] + [shortest + int((longest - shortest) * ((0.37 + _GOLDEN * i) % 1.0)) for i in range(1, n)]


def _q_lengths(c):
    if c["op"] in ("append", "paged"):
        return _lengths(c["seqs"], c["chunk"], 0 if c["empty"] else min(c["chunk"], 1))
    return _lengths(c["seqs"], c["q_len"], 0 if c["empty"] else 1)


def _k_lengths(c):
    if c["op"] in ("append", "paged"):  # the cache with the chunk in it: at least the chunk
        q = _q_lengths(c)
        return [max(a, b) for a, b in zip(_lengths(c["seqs"], c["k_len"]), q)]
    return _q_lengths(c) if c["k_len"] == 0 else list(reversed(_lengths(c["seqs"], c["k_len"])))


def _visible(c):
    """Number of (query, key) pairs of one head."""
    total = 0
    for q, k in zip(_q_lengths(c), _k_lengths(c)):
        if not c["causal"]:
            total += q * k
        else:  # query i sees keys 0 .. k - q + i
            m = min(q, k)  # rows that see anything see k - m + 1 .. k keys
            total += m * (k - m) + m * (m + 1) // 2
    return total


def listed():
    return [
        # q and k of a 21-frame 480p clip, 12 heads of 128: rotary positions over (frame, row, column), tensors stored head by head as
        # the Monarch attention takes them
        dict(name="rotary-480p", op="rotary", tokens=21 * 30 * 52, heads=12, kv_heads=12, d=128, pairs="22,21,21", interleaved=True,
             scaling="none", far=0, grid="21,30,52", dtype="bf16", backward=False, order="head"),
        # the gradient of a long float32 sequence's rotary positions: half layout on two thirds of the head, frequencies scaled by
        # band, positions around a million
        dict(name="rotary-back-f32", op="rotary", tokens=5003, heads=10, kv_heads=2, d=96, pairs="32", interleaved=False,
             scaling="bands", far=1_000_000, grid="", dtype="f32", backward=True, order="token"),
        # one token each of 24 sequences into pages of 16: the smallest call of a serving step
        dict(name="append-token", op="append", seqs=24, chunk=1, k_len=900, kv_heads=4, heads=12, d=64, page=16, pairs="32",
             interleaved=False, scaling="none", dtype="bf16", empty=False),
        # two new frames of 28 x 52 for each of 3 streams of video, one frame a page, three position axes' worth of pairs on one
        dict(name="append-frames", op="append", seqs=3, chunk=2 * 28 * 52, k_len=6 * 28 * 52, kv_heads=12, heads=12, d=128, page=28 * 52,
             pairs="64", interleaved=True, scaling="linear", dtype="bf16", empty=False),
        # a token each for five short sequences: where latency is all
        dict(name="paged-token-short", op="paged", seqs=5, chunk=1, k_len=700, kv_heads=4, heads=12, d=64, page=16, causal=True,
             dtype="bf16", empty=False),
        # a token each for 16 sequences of up to 16,384, 40 heads on 8: the cache read once
        dict(name="paged-token-long", op="paged", seqs=16, chunk=1, k_len=16384, kv_heads=8, heads=40, d=128, page=64, causal=True,
             dtype="bf16", empty=False),
        # a new frame of 15 x 26 tokens over up to 21 frames in pages of a frame; tokens of a frame see each other
        dict(name="paged-frame", op="paged", seqs=3, chunk=390, k_len=21 * 390, kv_heads=12, heads=12, d=128, page=390, causal=False,
             dtype="bf16", empty=False),
        # a dozen short ragged prompts, one of them empty, grouped heads of 64
        dict(name="packed-short", op="packed", seqs=12, q_len=700, k_len=0, kv_heads=4, heads=12, d=64, causal=True, dtype="bf16",
             empty=True, order="token"),
        # one whole prompt of 16,384 tokens, causal, 12 heads on 4
        dict(name="packed-16k", op="packed", seqs=1, q_len=16384, k_len=0, kv_heads=4, heads=12, d=128, causal=True, dtype="bf16",
             empty=False, order="token"),
        # float32, as a model is checked in full precision: ragged, odd sizes
        dict(name="packed-f32", op="packed", seqs=4, q_len=1001, k_len=0, kv_heads=2, heads=10, d=64, causal=True, dtype="f32",
             empty=False, order="token"),
        # training on three packed causal sequences of up to 4096, forward and backward
        dict(name="train-4k", op="train", seqs=3, q_len=4096, k_len=0, kv_heads=4, heads=12, d=128, causal=True, dtype="bf16",
             empty=False, order="token"),
        # training of the cross attention from ragged clips to text of up to 512 tokens, heads of 64, stored head by head
        dict(name="train-cross-d64", op="train", seqs=4, q_len=3157, k_len=512, kv_heads=10, heads=10, d=64, causal=False, dtype="bf16",
             empty=False, order="head"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    kv = rng.choice([1, 2, 4, 5, 8, 12])
    group = rng.choice([1, 1, 2, 3, 4, 5, 8])
    return kv, kv * group


def _pairs(rng, d, axes):
    part = rng.choice([d // 2, d // 2, d // 2, max(axes, 8 * (d // 32)), max(axes, d // 3)])
    if axes == 1:
        return str(part)
    side = part // 3
    return "%d,%d,%d" % (part - 2 * side, side, side)


def draw(rng):
    op = rng.choice(["rotary", "append", "paged", "paged", "packed", "packed", "train", "train"])
    most = {"f32": max(_weight(c) for c in listed() if c["dtype"] == "f32" and c["op"] != "rotary"),
            "bf16": max(_weight(c) for c in listed() if c["op"] == ("train" if op == "train" else "packed"))}
    while True:
        kv, heads = _heads(rng)
        c = dict(op=op, kv_heads=kv, heads=heads, d=rng.choice([64, 64, 128, 128, 128, 80, 96]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        if op == "rotary":
            axes = rng.choice([1, 3])
            c.update(pairs=_pairs(rng, c["d"], axes), interleaved=rng.random() < 0.5, scaling=rng.choice(["none", "linear", "bands"]),
                     far=rng.choice([0, 0, 1000, 1_000_000]), backward=rng.random() < 0.4, order=rng.choice(["token", "head"]), grid="")
            if axes == 3:
                t, y, x = rng.randint(1, 21), rng.randint(1, 30), rng.randint(1, 52)
                c.update(grid="%d,%d,%d" % (t, y, x), tokens=t * y * x, far=0)
            else:
                c.update(tokens=_log_int(rng, 1, 30000))
        elif op in ("append", "paged"):
            seqs = _log_int(rng, 1, 32)
            page = rng.choice([1, 7, 16, 16, 64, 64, 128, 390])
            chunk = 1 if rng.random() < 0.5 else _log_int(rng, 2, 1500)
            c.update(seqs=seqs, page=page, chunk=chunk, k_len=max(chunk, _log_int(rng, 1, 16384)), empty=rng.random() < 0.2)
            if op == "paged":
                c.update(causal=rng.random() < 0.6)
            else:
                c.update(pairs=_pairs(rng, c["d"], 1), interleaved=rng.random() < 0.5, scaling=rng.choice(["none", "linear", "bands"]))
        else:
            n = _log_int(rng, 1, 16)
            c.update(seqs=n, q_len=_log_int(rng, 1, 12000), k_len=0 if rng.random() < 0.7 else _log_int(rng, 1, 6000),
                     causal=rng.random() < 0.7, empty=rng.random() < 0.2, order=rng.choice(["token", "head"]))
            # the plain form holds all heads' scores at once
            if heads * (sum(_q_lengths(c)) * sum(_k_lengths(c))) > 3.3e9:
                continue
            if op == "train" and heads * (sum(_q_lengths(c)) * sum(_k_lengths(c))) > 1.1e9:
                continue
        if op in ("append", "paged") and sum(_k_lengths(c)) * c["kv_heads"] * c["d"] * _bytes(c) > 5e8:
            continue
        if op == "paged" and c["seqs"] * heads * c["chunk"] * max(_k_lengths(c)) > 1e9:
            continue
        if op == "paged" and c["seqs"] * heads * max(_k_lengths(c)) * c["d"] > 2e9:
            continue
        if _weight(c) <= most[c["dtype"]]:
            return c


def _weight(c):
    w = work(c)
    return max(w["flops"], 400 * w["bytes"])


def work(case):
    """Each input read once, each output written once; the products of visible (query, key) pairs."""
    c, es = case, _bytes(case)
    if c["op"] == "rotary":
        rows = c["tokens"] * (c["heads"] + c["kv_heads"])
        n = sum(int(p) for p in c["pairs"].split(","))
        return {"bytes": 2 * rows * c["d"] * es + 4 * c["tokens"], "flops": 6 * rows * n}
    q, k = sum(_q_lengths(c)), sum(_k_lengths(c))
    if c["op"] == "append":
        return {"bytes": 4 * q * c["kv_heads"] * c["d"] * es, "flops": 6 * q * c["kv_heads"] * int(c["pairs"])}
    q_bytes, k_bytes = q * c["heads"] * c["d"] * es, k * c["kv_heads"] * c["d"] * es
    product = 2 * c["d"] * c["heads"] * _visible(c)
    if c["op"] == "train":  # q k v out d_out dq dk dv, the log-sum-exp; two products forward, five backward
        return {"bytes": 4 * q_bytes + 4 * k_bytes + 4 * q * c["heads"], "flops": 7 * product}
    return {"bytes": 2 * q_bytes + 2 * k_bytes, "flops": 2 * product}


# ---- inputs -------------------------------------------------------------------------------------------------------------------


def _tokens(g, n, heads, d, dtype, order, deviation=1.0):
    """[n, heads, d], stored token by token or head by head."""
    x = torch.randn((heads, n, d) if order == "head" else (n, heads, d), generator=g, device="cuda") * deviation
    x = x.to(dtype)
    return x.transpose(0, 1) if order == "head" else x


def _starts(lengths):
    s = [0]
    for n in lengths:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


BASE, FACTOR, CONTEXT, LOW, HIGH = 10000.0, 8.0, 8192.0, 1.0, 32.0  # rotary base; a context stretched eightfold


def _scaling(case):
    """Arguments of the scaled frequencies: factor, context, turns below which all / above which nothing is stretched; amplitude."""
    if case["scaling"] == "none":
        return 1.0, 0.0, 0.0, 0.0, 1.0
    if case["scaling"] == "linear":
        return FACTOR, 0.0, 0.0, 0.0, 1.0
    return FACTOR, CONTEXT, LOW, HIGH, 1.2


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = _types(c)
    st = dict(case=c)
    if c["op"] in ("rotary", "append"):
        st["scaling"] = _scaling(c)
        st["pairs"] = [int(p) for p in c["pairs"].split(",")]
        if own:  # the plan of a model's rotary positions: its frequencies, kept by the program
            from paper_2601_22275_amd import binding
            factor, context, low, high, amplitude = st["scaling"]
            st["plan"] = binding.rotary_plan(st["pairs"], base=BASE, interleaved=c["interleaved"], factor=factor, context=context,
                                             low_turns=low, high_turns=high, amplitude=amplitude)
    if c["op"] == "rotary":
        n = c["tokens"]
        st["q"] = _tokens(g, n, c["heads"], c["d"], dtype, c["order"])
        st["k"] = _tokens(g, n, c["kv_heads"], c["d"], dtype, c["order"])
        at = torch.arange(n, device="cuda")
        if c["grid"]:
            _, y, x = (int(v) for v in c["grid"].split(","))
            pos = torch.stack([at // (y * x), at // x % y, at % x])
        else:
            pos = (at + c["far"] + int(torch.randint(0, 1000, (1,), generator=g, device="cuda")) * (c["far"] > 0))[None]
        st["positions"] = pos.to(torch.int32).contiguous()
        return st
    ql, kl = _q_lengths(c), _k_lengths(c)
    st["q_starts"] = _starts(ql)
    st["longest"] = (max(ql), max(kl))
    if c["op"] in ("append", "paged"):
        per = [-(-n // c["page"]) for n in kl]
        pages = sum(per) + 3  # a few pages nobody owns
        shape = (pages, c["page"], c["kv_heads"], c["d"])
        st["cache_k"] = torch.randn(shape, generator=g, device="cuda").to(dtype)
        st["cache_v"] = torch.randn(shape, generator=g, device="cuda").to(dtype)
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros((c["seqs"], max(per)), dtype=torch.int32, device="cuda")
        at = 0
        for s, n in enumerate(per):
            table[s, :n] = order[at:at + n]
            at += n
        st["table"], st["lengths"] = table, torch.tensor(kl, dtype=torch.int32, device="cuda")
        if c["op"] == "append":
            st["k"] = _tokens(g, sum(ql), c["kv_heads"], c["d"], dtype, "token")
            st["v"] = _tokens(g, sum(ql), c["kv_heads"], c["d"], dtype, "token")
            st["positions"] = torch.cat([torch.arange(b - a, b) for a, b in zip(ql, kl)]).to(torch.int32).cuda()[None].contiguous()
        else:
            st["q"] = _tokens(g, sum(ql), c["heads"], c["d"], dtype, "token", 1.5)
        return st
    if c["k_len"] != 0:
        st["k_starts"] = _starts(kl)
    else:
        st["k_starts"] = st["q_starts"]
    # logits with a deviation of about 2
    st["q"] = _tokens(g, sum(ql), c["heads"], c["d"], dtype, c["order"], 1.5)
    st["k"] = _tokens(g, sum(kl), c["kv_heads"], c["d"], dtype, c["order"], 1.3)
    st["v"] = _tokens(g, sum(kl), c["kv_heads"], c["d"], dtype, c["order"])
    if c["op"] == "train":
        st["d_out"] = _tokens(g, sum(ql), c["heads"], c["d"], dtype, c["order"])
    return st


# ---- the plain forms ----------------------------------------------------------------------------------------------------------


def _frequencies(st):
    out = []
    for n in st["pairs"]:
        out.append(BASE ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n))
    f = torch.cat(out)
    factor, context, low, high, _ = st["scaling"]
    if context == 0.0:
        return f / factor
    keep = ((context * f / (2 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
    return f * (keep + (1.0 - keep) / factor)


def _angles(st):
    axis = torch.cat([torch.full((n,), a, device="cuda") for a, n in enumerate(st["pairs"])])
    return st["positions"].double()[axis].transpose(0, 1) * _frequencies(st)  # [tokens, pairs]


def _rotated(x, cos, sin, interleaved):
    """x [tokens, heads, d] in 32 bits; cos, sin [tokens, 1, pairs]"""
    n = cos.shape[-1]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    u, w = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([u, w], dim=-1).flatten(-2) if interleaved else torch.cat([u, w], dim=-1)
    return torch.cat([turned, x[..., 2 * n:]], dim=-1)


def _plain_rotary(st):
    c = st["case"]
    angle, amplitude = _angles(st), st["scaling"][4]
    cos, sin = (amplitude * angle.cos()).float()[:, None], (amplitude * angle.sin()).float()[:, None]
    if c["op"] == "rotary" and c["backward"]:
        sin = -sin
    return tuple(_rotated(st[x].float(), cos, sin, c["interleaved"]).to(_types(c)) for x in (("q", "k") if c["op"] == "rotary" else ("k",)))


def _sequence_of(starts, n):
    """The sequence of each of n packed tokens, and the token's number in it."""
    at = torch.arange(n, device="cuda")
    s = (at[:, None] >= starts[None, 1:]).sum(1)
    return s, at - starts[s]


def _plain_append(st):
    c = st["case"]
    (k,) = _plain_rotary(st)
    s, i = _sequence_of(st["q_starts"], k.shape[0])
    new = st["q_starts"][1:] - st["q_starts"][:-1]
    at = (st["lengths"] - new)[s] + i
    page, slot = st["table"][s, at // c["page"]].long(), at % c["page"]
    st["cache_k"][page, slot] = k
    st["cache_v"][page, slot] = st["v"]
    return st["cache_k"], st["cache_v"]


def _weights(q, k, hidden, scale):
    """exp(logit - row maximum), their sums and the row maxima; a row that sees nothing has weights of zero."""
    s = torch.matmul(q, k.transpose(-2, -1).contiguous()).mul_(scale).masked_fill_(hidden, -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = s.sub_(m).exp_()
    return p, p.sum(-1, keepdim=True), m


def _by_head(x, group):
    x = x.float().transpose(0, 1).contiguous()
    return x[torch.arange(x.shape[0] * group, device="cuda") // group] if group > 1 else x


def _plain_packed(st):
    c = st["case"]
    group, scale = c["heads"] // c["kv_heads"], 1.0 / math.sqrt(c["d"])
    q, k, v = _by_head(st["q"], 1), _by_head(st["k"], group), _by_head(st["v"], group)
    qs, qi = _sequence_of(st["q_starts"], q.shape[1])
    ks, ki = _sequence_of(st["k_starts"], k.shape[1])
    hidden = qs[:, None] != ks[None]
    if c["causal"]:
        more = (st["k_starts"][1:] - st["k_starts"][:-1]) - (st["q_starts"][1:] - st["q_starts"][:-1])
        hidden |= ki[None] > (qi + more[qs])[:, None]
    p, l, m = _weights(q, k, hidden, scale)
    out = torch.matmul(p, v) / torch.where(l == 0, 1.0, l)
    y = out.transpose(0, 1).to(_types(c))
    if c["op"] == "packed":
        return y
    lse = (m + l.log())[..., 0]
    p /= torch.where(l == 0, 1.0, l)
    do = _by_head(st["d_out"], 1)
    dv = torch.matmul(p.transpose(-2, -1).contiguous(), do)
    ds = torch.matmul(do, v.transpose(-2, -1).contiguous())
    ds = ds.sub_((do * out).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-2, -1).contiguous(), q)
    dk, dv = (x.reshape(c["kv_heads"], group, -1, c["d"]).sum(1) for x in (dk, dv))
    return (y, lse) + tuple(x.transpose(0, 1).to(_types(c)) for x in (dq, dk, dv))


def _plain_paged(st):
    c = st["case"]
    group, scale = c["heads"] // c["kv_heads"], 1.0 / math.sqrt(c["d"])
    n, (most_q, most_k) = c["seqs"], st["longest"]
    new = st["q_starts"][1:] - st["q_starts"][:-1]
    i, j = torch.arange(most_q, device="cuda"), torch.arange(most_k, device="cuda")
    page = st["table"][:, j // c["page"]].long()
    own_head = torch.arange(c["heads"], device="cuda") // group
    k, v = (st[x][page, j % c["page"]][:, :, own_head].float().transpose(1, 2).contiguous() for x in ("cache_k", "cache_v"))
    at = (st["q_starts"][:-1, None] + i).clamp(max=st["q"].shape[0] - 1)
    q = st["q"][at].float().transpose(1, 2).contiguous()
    limit = st["lengths"][:, None] - (new[:, None] - 1 - i if c["causal"] else 0 * i)
    p, l, _ = _weights(q, k, (j >= limit[..., None])[:, None], scale)
    out = torch.matmul(p, v) / torch.where(l == 0, 1.0, l)
    s, at = _sequence_of(st["q_starts"], st["q"].shape[0])
    return out[s, :, at].to(_types(c))


def run(state):
    st = state
    c = st["case"]
    if not own:
        return {"rotary": _plain_rotary, "append": _plain_append, "paged": _plain_paged}.get(c["op"], _plain_packed)(st)
    from paper_2601_22275_amd import binding
    if c["op"] == "rotary":
        return binding.rotary(st["q"], st["k"], st["positions"], st["plan"], backward=c["backward"])
    if c["op"] == "append":
        binding.paged_append(st["k"], st["v"], st["cache_k"], st["cache_v"], st["table"], st["q_starts"], st["lengths"],
                             plan=st["plan"], positions=st["positions"])
        return st["cache_k"], st["cache_v"]
    if c["op"] == "paged":
        return binding.paged_attention(st["q"], st["cache_k"], st["cache_v"], st["table"], st["q_starts"], st["lengths"],
                                       causal=c["causal"])
    if c["op"] == "packed":
        return binding.packed_attention(st["q"], st["k"], st["v"], st["q_starts"], st["k_starts"], causal=c["causal"])
    out, lse = binding.packed_attention(st["q"], st["k"], st["v"], st["q_starts"], st["k_starts"], causal=c["causal"], lse=True)
    dq, dk, dv = binding.packed_attention_bwd(st["q"], st["k"], st["v"], out, st["d_out"], lse, st["q_starts"], st["k_starts"],
                                              causal=c["causal"])
    return out, lse, dq, dk, dv


# ---- 64 bits, from the definitions ----------------------------------------------------------------------------------------------


def _turn64(x, st):
    """Rotation as a product of complex numbers."""
    c = st["case"]
    factor, context, low, high, amplitude = st["scaling"]
    rows = []
    for a, n in enumerate(st["pairs"]):
        for i in range(n):
            f = BASE ** (-i / n)
            if context > 0.0:
                keep = min(1.0, max(0.0, (context * f / (2.0 * math.pi) - low) / (high - low)))
                f = f * keep + f * (1.0 - keep) / factor
            else:
                f = f / factor
            rows.append(st["positions"][a].double() * f)
    angle = torch.stack(rows, dim=1)
    if c.get("backward"):
        angle = -angle
    z = torch.polar(torch.full_like(angle, amplitude), angle)[:, None, :]
    n = angle.shape[1]
    x = x.double().contiguous().clone()
    even, odd = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if c["interleaved"] else (slice(0, n), slice(n, 2 * n))
    turned = torch.complex(x[..., even].contiguous(), x[..., odd].contiguous()) * z
    x[..., even], x[..., odd] = turned.real, turned.imag
    return x


def _one_head64(q, k, v, scale, causal, do=None):
    """One head of one sequence: out, lse and, with d_out, the gradients."""
    nq, nk = q.shape[0], k.shape[0]
    s = (q @ k.t()) * scale
    if causal:
        above = torch.ones(nq, nk, dtype=torch.bool, device=q.device).triu(nk - nq + 1)
        s = s.masked_fill(above, -math.inf)
    lse = torch.logsumexp(s, dim=1) if nk else torch.full((nq,), -math.inf, dtype=q.dtype, device=q.device)
    p = torch.where(torch.isfinite(lse)[:, None], torch.exp(s - lse[:, None]), torch.zeros_like(s))
    out = p @ v
    if do is None:
        return out, lse
    dp = do @ v.t()
    ds = p * (dp - (p * dp).sum(1, keepdim=True))
    return out, lse, scale * (ds @ k), scale * (ds.t() @ q), p.t() @ do


def exact(case, seed):
    c = case
    st = prepare(case, seed)
    if c["op"] == "rotary":
        return _turn64(st["q"], st), _turn64(st["k"], st)
    ql, kl = _q_lengths(c), _k_lengths(c)
    if c["op"] == "append":
        ck, cv = st["cache_k"].double(), st["cache_v"].double()
        k = _turn64(st["k"], st)
        table, at = st["table"].tolist(), 0
        for s in range(c["seqs"]):
            for p in range(kl[s] - ql[s], kl[s]):
                if p % c["page"] == 0 or p == kl[s] - ql[s]:  # a run of slots in one page
                    run_ = min(c["page"] - p % c["page"], kl[s] - p)
                    lo = p % c["page"]
                    ck[table[s][p // c["page"]], lo:lo + run_] = k[at:at + run_]
                    cv[table[s][p // c["page"]], lo:lo + run_] = st["v"][at:at + run_].double()
                    at += run_
        return ck, cv
    group, scale = c["heads"] // c["kv_heads"], 1.0 / math.sqrt(c["d"])
    out = torch.zeros(sum(ql), c["heads"], c["d"], dtype=torch.float64, device="cuda")
    if c["op"] == "train":
        lse = torch.zeros(c["heads"], sum(ql), dtype=torch.float64, device="cuda")
        dq = torch.zeros_like(out)
        dk = torch.zeros(sum(kl), c["kv_heads"], c["d"], dtype=torch.float64, device="cuda")
        dv = torch.zeros_like(dk)
    qa = ka = 0
    for s in range(c["seqs"]):
        q = st["q"][qa:qa + ql[s]].double()
        if c["op"] == "paged":
            pages = st["table"][s, :-(-kl[s] // c["page"])].long()
            k, v = (st[x][pages].flatten(0, 1)[:kl[s]].double() for x in ("cache_k", "cache_v"))
        else:
            k, v = st["k"][ka:ka + kl[s]].double(), st["v"][ka:ka + kl[s]].double()
        for h in range(c["heads"]):
            head = (q[:, h].contiguous(), k[:, h // group].contiguous(), v[:, h // group].contiguous(), scale, c["causal"])
            if c["op"] != "train":
                out[qa:qa + ql[s], h] = _one_head64(*head)[0]
                continue
            y, l, a, b, w = _one_head64(*head, st["d_out"][qa:qa + ql[s], h].double())
            out[qa:qa + ql[s], h], lse[h, qa:qa + ql[s]], dq[qa:qa + ql[s], h] = y, l, a
            dk[ka:ka + kl[s], h // group] += b
            dv[ka:ka + kl[s], h // group] += w
        qa, ka = qa + ql[s], ka + kl[s]
    return (out, lse, dq, dk, dv) if c["op"] == "train" else out
