"""Plain implementations, in 64 bits and from the definitions, of the router,
the combine's backward pass and the 8-bit products: what the GPU tests of these
operators compare with."""
from __future__ import annotations

import math

import numpy as np

U32 = 2.0 ** -24   # rounding to fp32: largest relative error
U16 = 2.0 ** -8    # rounding to bf16, 8 significant bits (1 + 2^-8 goes to 1)


def bf16_bits(f):
    """fp32 array -> bf16 patterns, to nearest-even, NaN to 0x7FC0."""
    f = np.ascontiguousarray(f, np.float32)
    b = f.view(np.uint32).astype(np.uint64)
    out = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(f), np.uint16(0x7FC0), out)


def from_bits(b):
    return (np.ascontiguousarray(b, np.uint16).astype(np.uint32) << 16).view(np.float32)


def bf16(f):
    """fp32 array rounded to bf16, as fp32."""
    return from_bits(bf16_bits(f))


def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1.0 + e)


def scores(z, kind):
    """s and p of one token's logits (-inf allowed, one at least above it)."""
    if kind == "sigmoid":
        c = min(z.max(), 0.0)
        u = np.exp(np.minimum(z, 0.0) - c) / (1.0 + np.exp(-np.abs(z)))
        return sigmoid(z), u / u.sum()
    u = np.exp(z - z.max())
    return u / u.sum(), u / u.sum()


def keys(z, r, bias):
    """Selection keys: softmax z + bias in fp32, sigmoid s + bias in 64 bits."""
    if r["score"] == "sigmoid" and (bias is not None or r["n_group"]):
        k = sigmoid(z.astype(np.float64)) + (0.0 if bias is None else bias.astype(np.float64))
    else:
        k = (z + (np.float32(0) if bias is None else bias)).astype(np.float32).astype(np.float64)
    return np.where(np.isneginf(z), -np.inf, k)


def select(z, r, bias):
    """The k ids of one token's fp32 logits, -1 where none is left."""
    key = keys(z, r, bias)
    E, G = len(z), r["n_group"]
    if G:
        size = E // G
        two = np.sort(key.reshape(G, size), axis=1)[:, -2:]
        s = two[:, 0] + two[:, 1]
        best = sorted(range(G), key=lambda g: (-s[g], g))[:r["top_group"]]
        key = np.array([key[e] if e // size in best else -np.inf for e in range(E)])
    order = sorted((e for e in range(E) if key[e] > -np.inf), key=lambda e: (-key[e], e))[:r["k"]]
    return np.array(order + [-1] * (r["k"] - len(order)), np.int32)


def gates(z, ids, r):
    """Gates of one token: from the chosen logits alone where renormalised."""
    g = np.zeros(len(ids))
    on = [i for i, e in enumerate(ids) if e >= 0 and z[e] > -np.inf]
    if not on:
        return g
    zi = z[[ids[i] for i in on]].astype(np.float64)
    if r["renorm"]:
        low = np.minimum(zi, 0.0) if r["score"] == "sigmoid" else zi
        u = np.exp(low - low.max())
        if r["score"] == "sigmoid":
            u = u / (1.0 + np.exp(-np.abs(zi)))
        g[on] = u / u.sum() * r["scale"]
    else:
        g[on] = scores(z.astype(np.float64), r["score"])[0][[ids[i] for i in on]] * r["scale"]
    return g


def route(z, r, bias=None, mask=None):
    """ids [T][k], gates, counts / sums of p / tokens by sequence."""
    T, E = z.shape
    L = r["seq_len"] or max(T, 1)
    n = max(1, math.ceil(T / L))
    ids = np.full((T, r["k"]), -1, np.int32)
    gate = np.zeros((T, r["k"]))
    counts, tokens = np.zeros((n, E), np.int64), np.zeros(n, np.int64)
    psum = np.zeros((n, E))
    for t in range(T):
        if (mask is not None and not mask[t]) or not (z[t] > -np.inf).any():
            continue
        ids[t] = select(z[t], r, bias)
        if ids[t, 0] < 0:
            continue
        gate[t] = gates(z[t], ids[t], r)
        np.add.at(counts[t // L], ids[t][ids[t] >= 0], 1)
        tokens[t // L] += 1
        psum[t // L] += scores(z[t].astype(np.float64), r["score"])[1]
    return ids, gate, counts, psum, tokens


def balance(counts, load_tokens, psum, tokens, r, alpha):
    n, E = counts.shape
    coef = np.zeros((n, E))
    for s in range(n):
        if load_tokens[s] > 0 and tokens[s] > 0:
            coef[s] = alpha * E * counts[s] / (n * r["k"] * float(load_tokens[s]) * float(tokens[s]))
    return float((coef * psum).sum()), coef


def objective(z, ids, r, dgate, w):
    """What the router's gradient is the gradient of, for one token:
    sum dgate * gate + sum w * p."""
    return float((dgate * gates(z, ids, r)).sum() + (w * scores(z, r["score"])[1]).sum())


def route_grad(z, ids, r, dgate, w):
    """The gradient by the formula, for one token's 64-bit logits, and a bound on
    the sums of magnitudes that its elements are made of."""
    s, p = scores(z, r["score"])
    dz = p * (w - (w * p).sum())
    mag = p * (np.abs(w) + (np.abs(w) * p).sum())
    if r["score"] == "sigmoid":
        dz = dz * (1.0 - s)
    on = [i for i, e in enumerate(ids) if e >= 0 and z[e] > -np.inf]
    if on:
        e = np.array([ids[i] for i in on])
        dg = dgate[on] * r["scale"]
        if r["renorm"]:
            q = gates(z, ids[on], {**r, "scale": 1.0})
            d, m = q * (dg - (q * dg).sum()), q * (np.abs(dg) + (q * np.abs(dg)).sum())
        else:
            d, m = s[e] * dg, s[e] * np.abs(dg)
        if r["score"] == "sigmoid":
            d = d * (1.0 - s[e])
        elif not r["renorm"]:
            dz = dz - p * d.sum()
            mag = mag + p * m.sum()
        np.add.at(dz, e, d)
        np.add.at(mag, e, m)
    dead = np.isneginf(z)
    return np.where(dead, 0.0, dz), np.where(dead, 0.0, mag)


def quant_rows(x):
    """q, scale of fp32 rows, each operation rounded to fp32."""
    x = np.ascontiguousarray(x, np.float32)
    a = np.abs(x).max(axis=1) if x.shape[1] else np.zeros(len(x), np.float32)
    finite = np.isfinite(x).all(axis=1)
    live = finite & (a > np.float32(2.0 ** -100))
    one = np.where(live, a, np.float32(1))
    inv = np.where(live, np.float32(127) / one, np.float32(0)).astype(np.float32)
    q = np.rint(np.where(live[:, None], x, np.float32(0)) * inv[:, None]).astype(np.int8)
    scale = np.where(live, one / np.float32(127), np.where(finite, 0.0, np.nan)).astype(np.float32)
    return q, scale


def expert_matmul(xq, xs, wq, ws, off, of, act):
    """y in 64 bits, and a bound on its relative rounding error in fp32."""
    N = wq.shape[1]
    y = np.zeros((len(xq), N // 2 if act else N))
    rel = np.zeros_like(y)
    for g in range(len(off) - 1):
        lo, hi = off[g], off[g + 1]
        if hi <= lo:
            continue
        w = of[g] if of is not None else g
        v = (xq[lo:hi].astype(np.float64) @ wq[w].T.astype(np.float64)) * xs[lo:hi, None].astype(np.float64) \
            * ws[w].astype(np.float64)
        if act:
            a, b = v[:, :N // 2], v[:, N // 2:]
            y[lo:hi] = a * sigmoid(a) * b
            # 3 roundings of each product; exp's argument carries |a| of them; 8 more
            # for exp (2), the sum, the quotient, silu's rounding, the product
            rel[lo:hi] = (14 + 3 * np.abs(a)) * U32
        else:
            y[lo:hi], rel[lo:hi] = v, 3.01 * U32
    return y, rel
