"""References of the operators in 64 bits, and how far a correct implementation may be from them."""
import math

import numpy as np


def bf16(x):
    """float64 values rounded to bf16 (nearest, ties to even) and back."""
    import synth
    return synth.bf16_to_f32(synth.bf16_round(np.asarray(x, dtype=np.float32))).astype(np.float64).reshape(np.shape(x))


def w4_plain(rng, n, k, group, exact=False):
    """Random codes [n][k/2] and scales (bf16 bits) [n][k/group] in plain order, and the matrix they stand for."""
    import synth
    c = rng.integers(0, 16, size=(n, k), dtype=np.uint8)
    s = 2.0 ** rng.integers(-3, 1, size=(n, k // group)) if exact else rng.uniform(0.02, 0.2, size=(n, k // group))
    bits = synth.bf16_round(s.astype(np.float32)).reshape(s.shape)
    w = (c.astype(np.float64) - 8) * np.repeat(synth.bf16_to_f32(bits).astype(np.float64), group, axis=1)
    return (c[:, 0::2] | c[:, 1::2] << 4), bits, w


def w4_matrix(codes, bits, group):
    """The matrix of plain-order codes and scales."""
    import synth
    c = np.empty((codes.shape[0], 2 * codes.shape[1]))
    c[:, 0::2], c[:, 1::2] = codes & 15, codes >> 4
    return (c - 8) * np.repeat(synth.bf16_to_f32(bits).astype(np.float64), group, axis=1)


def gelu(v):
    return v * 0.5 * (1 + np.vectorize(math.erf, otypes=[float])(v / math.sqrt(2)))


def act(v, name):
    return gelu(v) if name == "gelu" else np.maximum(v, 0) if name == "relu" else v


def w4_tolerance(x, w, y, f32):
    """Elementwise. One rounding of the result (bf16 half a step: 2^-8 of it; fp32 2^-24). fp32 sums: K products and about as
    many of the surplus, each addition off by at most 2^-23 (the matrix cores may truncate) of a partial
    sum, whose rms is below 31 + 24 = 55 times that of the terms without their codes, sqrt(sum (s x)^2); K of them
    add up as a walk of sqrt(K) steps. (s x)^2 is bounded by (w x)^2's rows with the code's 8 taken as the mean
    square 21.25 of a uniform code. Factor 4 over the rms for the largest of up to 10^6 outputs. GELU's formula
    adds 1.5e-7 of the argument (and has a slope of at most 1.13)."""
    k = x.shape[1]
    walk = np.sqrt((x * x) @ (w * w).T / 21.25)
    return 4 * 2.0 ** -23 * math.sqrt(k) * 55 * walk * 1.13 + np.abs(y) * (2.0 ** -24 if f32 else 2.0 ** -8) + 3e-7 * (1 + np.abs(y))


def seen(qn, kn, causal, left, right, sinks):
    """[qn][kn] truth values: which keys each query sees."""
    p = np.arange(qn)[:, None] + (kn - qn)
    j = np.arange(kn)[None]
    near = np.ones((qn, kn), dtype=bool)
    if left >= 0:
        near &= j >= p - left
    if right >= 0:
        near &= j <= p + right
    m = near | (j < sinks)
    return m & (j <= p) if causal else m


def attention(q, k, v, m, scale):
    """One sequence's head: q [qn][d], k, v [kn][d], m [qn][kn] -> (out, tolerance). The tolerance, elementwise: the
    exponentials are rounded to bf16 (2^-8 of each at most) before they multiply v, the output once more (2^-8 of it); scores,
    exponentials and sums are fp32: a dot product of d terms is off by at most d 2^-23 of sum |q k|, which
    moves an exponential by as much of itself, and the hardware exponential, the running rescaling and the sums add less than 1e-5."""
    out, tol = np.zeros((q.shape[0], v.shape[1])), np.zeros((q.shape[0], v.shape[1]))
    if k.shape[0] == 0:
        return out, tol
    with np.errstate(invalid="ignore"):
        s = np.where(m, (q @ k.T) * scale, -np.inf)
    some = m.any(axis=1)
    top = np.where(some, np.max(s, axis=1), 0)
    e = np.where(m, np.exp(s - top[:, None]), 0)
    w = e / np.where(some, e.sum(axis=1), 1)[:, None]
    out[some] = (w @ v)[some]
    spread = float(np.max((np.abs(q) @ np.abs(k).T) * scale)) if m.any() else 0.0
    small = 1e-5 + 2 * q.shape[1] * 2.0 ** -23 * spread
    tol = 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + small) * (1 + 2.0 ** -8) * (w @ np.abs(v)) + 1e-30
    return out, tol
