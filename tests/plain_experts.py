"""Plain implementations, in 64 bits and from the definitions, of the experts'
products in bf16 with their gradients and in 8-bit floating point: what their
tests compare with.  Each product comes with a bound on the error of an fp32
evaluation: a sum of n terms, in any order, is off by at most n roundings of the
sum of their magnitudes, counted twice since the matrix unit may round down."""
from __future__ import annotations

import numpy as np

from plain64 import U16, U32, sigmoid

def matmul(a, b):
    """a @ b in 64 bits; by torch where the GPU is at hand, since large ones take long."""
    if a.size * b.shape[1] > 1 << 26:
        import torch
        if torch.cuda.is_available():
            return (torch.from_numpy(np.ascontiguousarray(a)).cuda() @ torch.from_numpy(np.ascontiguousarray(b)).cuda()).cpu().numpy()
    return a @ b


TINY = 1e-34   # below this the fast exponential may give 0


def silu(a):
    return a * sigmoid(a)


def swiglu(v):
    a, b = np.split(v, 2, axis=1)
    return silu(a) * b


def swiglu_grad(v, pre):
    a, b = np.split(pre, 2, axis=1)
    s = sigmoid(a)
    return np.concatenate([v * b * s * (1 + a * (1 - s)), v * a * s], axis=1)


def activate(v, dv, act, pre=None):
    """The result of rows v that are off by at most dv, and a bound on its error in fp32
    (14 operations and the exponential, whose argument carries 3 |a| roundings)."""
    with np.errstate(invalid="ignore", over="ignore"):
        if act == "none":
            return v, dv
        if act == "swiglu":
            a, b = np.split(v, 2, axis=1)
            da, db = np.split(dv, 2, axis=1)
            y = silu(a) * b
            # |silu'| < 1.1, and da itself is far below 1
            return y, 1.1 * da * (np.abs(b) + db) + np.abs(silu(a)) * db + (16 + 3 * np.abs(a)) * U32 * np.abs(y) \
                + TINY * (1 + np.abs(b))
        a, b = np.split(pre, 2, axis=1)
        s = sigmoid(a)
        y = swiglu_grad(v, pre)
        size = np.concatenate([np.abs(b) * s * (1 + np.abs(a) * (1 - s)), np.abs(a) * s], axis=1)
        a2, v2, dv2 = (np.concatenate([t, t], axis=1) for t in (a, v, dv))
        return y, size * (dv2 + (20 + 3 * np.abs(a2)) * U32 * np.abs(v2)) + TINY * (1 + np.abs(v2))


def rounded(y, err, f32):
    """The bound with the rounding of the result (half a step of its type)."""
    u = U32 if f32 else U16
    return err + u * (np.abs(y) + err) + 1e-37


def eights(x):
    """The largest magnitude of each 8 neighbours of the last axis."""
    x = np.pad(np.abs(x), [(0, 0)] * (x.ndim - 1) + [(0, -x.shape[-1] % 8)])
    return x.reshape(*x.shape[:-1], -1, 8).max(axis=-1)


def product(x, w, off, of, act, trans=False, pre=None, cut=False, taken_to_bf16=False):
    """y [M], its bound, v and its bound, of rows x [M][K] (fp64) and weights
    [n_w][N][K] (trans: [n_w][K][N]); rows outside the blocks are NaN.
    cut: by the matrix unit's 8-bit products, 8 neighbours of which are cut 13 bits
    below the exponent of the largest before they are added: each of the 7 others
    loses less than 2^-13 of it.
    taken_to_bf16: values below 2^-126 are off by half of bf16's least step, 2^-133."""
    M, K = x.shape
    N = w.shape[2] if trans else w.shape[1]
    width = {"none": N, "swiglu": N // 2, "swiglu_grad": 2 * N}[act]
    y, err = np.full((M, width), np.nan), np.full((M, width), np.nan)
    v, dv = np.full((M, N), np.nan), np.full((M, N), np.nan)
    sides = {}  # of each weight: itself, its magnitudes, their largest of 8
    for g in range(len(off) - 1):
        lo, hi = off[g], off[g + 1]
        if hi <= lo:
            continue
        j = of[g] if of is not None else g
        if j not in sides:
            ww = w[j] if trans else w[j].T
            sides[j] = ww, np.abs(ww), eights(ww.T).T if cut else None
        ww, size, most = sides[j]
        with np.errstate(invalid="ignore"):
            v[lo:hi] = matmul(x[lo:hi], ww)
            dv[lo:hi] = 2 * K * U32 * matmul(np.abs(x[lo:hi]), size) + 1e-37
            if cut:
                dv[lo:hi] += 7 * 2.0 ** -13 * matmul(eights(x[lo:hi]), most)
            if taken_to_bf16:
                small = (np.abs(x[lo:hi]) < 2.0 ** -126) & (x[lo:hi] != 0), (size < 2.0 ** -126) & (ww != 0)
                if small[0].any() or small[1].any():
                    dv[lo:hi] += 2.0 ** -134 * (small[0] @ size + np.abs(x[lo:hi]) @ small[1])
        y[lo:hi], err[lo:hi] = activate(v[lo:hi], dv[lo:hi], act, None if pre is None else pre[lo:hi])
    return y, err, v, dv


def weight_grad(dy, x, off, of, n_w):
    """dw [n_w][N][K] and its bound."""
    dw = np.zeros((n_w, dy.shape[1], x.shape[1]))
    mag, rows = np.zeros_like(dw), np.zeros(n_w)
    for g in range(len(off) - 1):
        lo, hi = off[g], off[g + 1]
        if hi <= lo:
            continue
        w = of[g] if of is not None else g
        dw[w] += matmul(dy[lo:hi].T, x[lo:hi])
        mag[w] += matmul(np.abs(dy[lo:hi]).T, np.abs(x[lo:hi]))
        rows[w] += hi - lo
    return dw, 2 * (rows[:, None, None] + 2) * U32 * mag + 1e-37


def e4m3_values():
    """The 256 values of e4m3 (bias 7, subnormals below 2^-6, 0x7F and 0xFF NaN)."""
    b = np.arange(256)
    e, m = b >> 3 & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where(b & 0x7F == 0x7F, np.nan, v)
    return np.where(b & 0x80, -v, v)


def e4m3_bits(v):
    """fp64 values of at most 448 in magnitude -> patterns, to nearest-even."""
    a = np.abs(v)
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    r = np.rint(a / step) * step
    table = e4m3_values()[:127]  # rising
    at = np.searchsorted(table, r)
    assert (table[at] == r).all()
    return (at | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def quant_blocks(x, ldq):
    """q [rows][ldq], scale [rows][pitch] of fp32 rows."""
    rows, K = x.shape
    q = np.zeros((rows, ldq), np.uint8)
    scale = np.zeros((rows, 4 * -(-K // 512)), np.uint8)
    for b in range(-(-K // 128)):
        part = x[:, b * 128:(b + 1) * 128].astype(np.float64)
        fine = np.isfinite(part).all(axis=1)
        part = np.where(fine[:, None], part, 0.0)
        m, p = np.frexp(np.abs(part).max(axis=1))
        e = np.where(m == 0, -127, np.maximum(p - 9 + (m > 0.875), -127))
        bits = e4m3_bits(part * 2.0 ** -e[:, None].astype(np.float64))
        q[:, b * 128:b * 128 + part.shape[1]] = np.where(fine[:, None], bits, 0x7F)
        scale[:, b] = np.where(fine, e + 127, 255)
    return q, scale


def dequantised(q, scale):
    """fp64 values of e4m3 rows [rows][K] and their scales' bytes."""
    K = q.shape[-1]
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return e4m3_values()[q] * np.repeat(s, 128, axis=-1)[..., :K]
