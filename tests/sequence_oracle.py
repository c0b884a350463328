"""Token-sequence operators in 64 bits (numpy), with element-wise bounds on what the kernels may be off by.

Bounds count roundings.  u: half a step of the stored type (bf16 2^-8, float32 2^-24); w: of a softmax weight or its gradient as a
matrix operand (2^-8 for bf16 tensors, none for float32).  A logit is a dot product of d terms in fp32, off by at most (d + 4) 2^-24 of the sum
of its terms' magnitudes (products, sums, scale, conversion to the exponent's base); an exponential by that, absolutely, relative to itself."""
import math

import numpy as np

U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def attention(q, k, v, scale, causal, dtype, d_out=None):
    """One head of one sequence.  Returns {name: (value, bound)} of out, lse and, with d_out, dq, dk, dv."""
    nq, d = q.shape
    nk = k.shape[0]
    u, w = U[dtype], 2.0 ** -8 if dtype == "bf16" else 0.0
    sees = np.ones((nq, nk), dtype=bool)
    if causal:
        sees = np.arange(nk)[None] <= (nk - nq + np.arange(nq))[:, None]
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        s = scale * (q @ k.T)
        s = np.where(sees, s, -np.inf)
        m = np.max(s, axis=1, initial=-np.inf)
        ref = np.where(np.isfinite(m), m, np.where(np.isneginf(m), 0.0, m))
        p = np.exp(s - ref[:, None])
        l = p.sum(1)
        p = np.where(l[:, None] == 0, 0.0, p / np.where(l == 0, 1.0, l)[:, None])
        lse = np.where(l == 0, -np.inf, ref + np.log(np.where(l == 0, 1.0, l)))
        out = np.zeros((nq, v.shape[1]))
        if np.isfinite(v).all():
            out = p @ v
        else:  # what a row does not see does not reach it
            for i in range(nq):
                out[i] = (p[i, sees[i], None] * v[sees[i]]).sum(0)
    if not (np.isfinite(q).all() and np.isfinite(k).all() and np.isfinite(v).all()):
        return {"out": (out, None), "lse": (lse, None)}
    e = (d + 4) * 2.0 ** -24 * scale * np.max(np.where(sees, np.abs(q) @ np.abs(k).T, 0.0), axis=1, initial=0.0) + 2.0 ** -22
    e = e + 2.0 ** -23 * (np.abs(np.where(np.isfinite(lse), lse, 0.0)) + 4)  # the reference and the exponent's argument
    spread = p @ np.abs(v)
    # a weight and their sum carry e and w each; sums of nk terms in fp32
    e_out = (2 * e + 2 * w + (nk + 8) * 2.0 ** -24)[:, None] * spread
    got = {"out": (out, e_out + u * (np.abs(out) + e_out) + 1e-30), "lse": (lse, np.where(np.isfinite(lse), 2 * e + 2.0 ** -22 + nk * 2.0 ** -24, 0.0))}
    if d_out is None:
        return got
    dp = d_out @ v.T
    delta = (d_out * out).sum(1)
    ds = p * (dp - delta[:, None])
    e_p = 4 * e + w  # P from the stored log-sum-exp
    e_dp = (d + 4) * 2.0 ** -24 * (np.abs(d_out) @ np.abs(v).T)
    e_delta = (np.abs(d_out) * (got["out"][1] + (d + 4) * 2.0 ** -24 * np.abs(out))).sum(1)
    e_ds = p * (e_dp + e_delta[:, None]) + np.abs(ds) * (4 * e + w + 2.0 ** -22)[:, None]
    dq, dk, dv = scale * ds @ k, scale * ds.T @ q, p.T @ d_out
    n = (max(nq, nk) + 8) * 2.0 ** -24
    b_dq = scale * (e_ds + n * np.abs(ds)) @ np.abs(k)
    b_dk = scale * (e_ds + n * np.abs(ds)).T @ np.abs(q)
    b_dv = ((e_p + n)[:, None] * p).T @ np.abs(d_out)
    got.update(dq=(dq, b_dq + u * (np.abs(dq) + b_dq) + 1e-30), dk=(dk, b_dk + 1e-30), dv=(dv, b_dv + 1e-30))  # dk, dv: rounded after the heads' sum
    return got


def packed(q, k, v, q_starts, k_starts, scale, causal, dtype, d_out=None):
    """All heads and sequences: {name: (value, bound)} in the calls' layouts; rows of no sequence are NaN."""
    heads, kv = q.shape[1], k.shape[1]
    u = U[dtype]
    names = ["out", "lse"] + ([] if d_out is None else ["dq", "dk", "dv"])
    shape = {"out": q.shape, "lse": (heads, q.shape[0]), "dq": q.shape, "dk": k.shape, "dv": v.shape}
    got = {n: [np.full(shape[n], np.nan), np.full(shape[n], 0.0)] for n in names}
    for s in range(len(q_starts) - 1):
        a, b, c, e = q_starts[s], q_starts[s + 1], k_starts[s], k_starts[s + 1]
        for n in ("dk", "dv"):
            if n in got:
                got[n][0][c:e] = 0.0
        for h in range(heads):
            g = h // (heads // kv)
            r = attention(q[a:b, h], k[c:e, g], v[c:e, g], scale, causal, dtype, None if d_out is None else d_out[a:b, h])
            for i in range(2):
                got["out"][i][a:b, h] = r["out"][i] if r["out"][i] is not None else np.nan
                got["lse"][i][h, a:b] = r["lse"][i] if r["lse"][i] is not None else np.nan
                if d_out is not None:
                    got["dq"][i][a:b, h] = r["dq"][i]
                    got["dk"][i][c:e, g] += r["dk"][i]
                    got["dv"][i][c:e, g] += r["dv"][i]
    for n in ("dk", "dv"):
        if n in got:
            got[n][1] += u * (np.abs(got[n][0]) + got[n][1]) + 1e-30
    return got


def frequencies(axis_pairs, base=10000.0, factor=1.0, context=0.0, low=0.0, high=0.0):
    f = np.concatenate([base ** (-np.arange(n) / n) for n in axis_pairs])
    if factor != 1.0:
        keep = np.zeros_like(f) if context == 0 else np.clip((context * f / (2 * math.pi) - low) / (high - low), 0, 1)
        f = f * (keep + (1 - keep) / factor)
    return f


def rotary(x, positions, axis_pairs, f, interleaved, backward=False, amplitude=1.0):
    """x [tokens, heads, d], positions [axes, tokens].  Returns the turned tensor."""
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    angle = positions.astype(np.float64)[axis].T * f
    c, s = amplitude * np.cos(angle)[:, None], amplitude * np.sin(angle)[:, None] * (-1 if backward else 1)
    n = len(f)
    y = x.astype(np.float64).copy()
    i0, i1 = (np.arange(n) * 2, np.arange(n) * 2 + 1) if interleaved else (np.arange(n), np.arange(n) + n)
    y[..., i0] = x[..., i0] * c - x[..., i1] * s
    y[..., i1] = x[..., i0] * s + x[..., i1] * c
    return y


def rotary_bound(x, y, axis_pairs, interleaved, amplitude, dtype):
    """One rounding of the result; sine, cosine (2^-22 absolute: the argument's rounding to 32 bits and the functions' own) and two products in fp32."""
    n = sum(axis_pairs)
    b = np.zeros_like(y)
    i0, i1 = (np.arange(n) * 2, np.arange(n) * 2 + 1) if interleaved else (np.arange(n), np.arange(n) + n)
    both = abs(amplitude) * (np.abs(x[..., i0]) + np.abs(x[..., i1]))
    b[..., i0] = b[..., i1] = 2.0 ** -21 * both
    b[..., :2 * n] += U[dtype] * (np.abs(y[..., :2 * n]) + b[..., :2 * n])
    return b + 1e-30
