"""8-bit integer rows, products and SwiGLU experts, and what stands between two blocks, from their
definitions.

A row's scale is a / 127, a its largest magnitude (2^-100 at least), a code its number times
127 / a rounded to an integer (ties to even); quotients and product are rounded to float32 first."""
from __future__ import annotations

import numpy as np

f32 = np.float32
LEAST = f32(2.0 ** -100)


def bf16_round(x):
    """float32 to the nearest bf16 number (ties to even), as float32."""
    x = np.ascontiguousarray(x, dtype=f32)
    b = x.view(np.uint32)
    r = ((b.astype(np.uint64) + 0x7fff + ((b >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(f32)
    return np.where(np.isfinite(x), r, x).astype(f32)


def bf16_step(v):
    """Distance of the bf16 numbers around |v| (the one above a power of two)."""
    a = np.maximum(np.abs(np.asarray(v, dtype=np.float64)), 2.0 ** -126)
    return 2.0 ** (np.floor(np.log2(a)) - 7)


def quantize_rows(x):
    """x [M, K] (numbers that float32 holds) -> codes int8, scales float32 [M]."""
    x = np.asarray(x, dtype=f32)
    fine = np.isfinite(x).all(1)
    v = np.where(fine[:, None], x, f32(0))
    a = np.maximum(np.abs(v).max(1), LEAST)
    q = np.rint(v * (f32(127) / a)[:, None]).astype(np.int8)
    return q, np.where(fine, a / f32(127), f32(np.nan)).astype(f32)


def product(x, xs, w, ws):
    """float64 results: exact sums of the codes' products times the scales."""
    sums = x.astype(np.float64) @ w.astype(np.float64).T      # (|sum| <= 2^28: exact)
    return sums * (xs.astype(np.float64)[:, None] * ws.astype(np.float64)[None, :])


PRODUCT_EPS = 3.1 * 2.0 ** -24      # the sum, the scales' product and the result rounded to fp32


def steepest(g, eg, sigma):
    """Largest |SiLU'| within eg of g, sigma the logistic function of g: |SiLU'(t)| <= sigma(t) (1 + |t|), at most 1.1
    anywhere, and sigma(t) <= sigma(g) e^|t - g|."""
    return np.minimum(1.1, sigma * np.exp(np.minimum(eg, 1.0)) * (1.0 + np.abs(g) + eg) + 1.1 * (eg > 1.0))


FAR = -87.0      # below it SiLU, less than 2^-119 there, may be taken as 0 (the reciprocal of 1 + e^-g is no normal number)


def swiglu_rows(x, xs, gate, up, down):
    """One expert (each weight a pair of codes and scales) on rows x, and how far a computation that
    follows the rounding points may be from it.

    g and u are off by PRODUCT_EPS of themselves, the activation by that times the steepest SiLU there and
    (|g| + 4) 2^-22 of itself.  Rounded to bf16 the error vanishes, except next to a border between
    two numbers, where it is a step; then rounded to 8 bits the same, except that a row whose largest
    number is itself in doubt may have another scale: then any value may move by a step.  A value of a gate
    below FAR may be anything down to 0."""
    g, u = product(x, xs, *gate), product(x, xs, *up)
    eg, eu = PRODUCT_EPS * np.abs(g), PRODUCT_EPS * np.abs(u)
    with np.errstate(over="ignore"):
        sigma = 1.0 / (1.0 + np.exp(-g))
    silu = g * sigma
    a = silu * u
    ea = steepest(g, eg, sigma) * eg * (np.abs(u) + eu) + np.abs(silu) * eu
    ea += (np.abs(g) + 4.0) * 2.0 ** -22 * np.abs(a) + 2.0 ** -140
    step = bf16_step(a)
    doubt = np.abs(np.abs(a / step - np.floor(a / step)) - 0.5) <= ea / step
    b = bf16_round(a).astype(np.float64)
    far = g - eg < FAR
    doubt |= far
    eb = np.where(doubt, step, 0.0) + np.where(far, np.abs(b), 0.0)
    q, qs = quantize_rows(b)
    s = qs.astype(np.float64)[:, None]
    at = b / s
    near = np.abs(np.abs(at - np.floor(at)) - 0.5) <= eb / s + 127 * 2.0 ** -22
    top = np.abs(b).max(1, keepdims=True)
    moving = (doubt & (np.abs(b) >= top - 2.0 * step)).any(1, keepdims=True)
    off = np.where(moving, 1.02 * s + eb, np.where(near, s + np.where(far, eb, 0.0), 0.0))
    y = product(q, qs, *down)
    w = np.abs(down[0].astype(np.float64)) * down[1].astype(np.float64)[:, None]
    return y, off @ w.T + PRODUCT_EPS * np.abs(y)


def inverse_rms(v, eps):
    """float32 1 / sqrt(mean v^2 + eps) of float32 rows."""
    return (1.0 / np.sqrt((v.astype(np.float64) ** 2).mean(1, keepdims=True) + np.float64(f32(eps)))).astype(f32)


def stream(x, y, w_post, gate, residual_scale, eps, wide):
    """The stream's new rows (float32, of its type) from float32 rows; x, y, w_post, gate None: not there.
    gate: a row for each row."""
    u = None
    if y is not None:
        u = y.astype(f32)
        if w_post is not None:
            u = u * inverse_rms(u, eps) * w_post
        if gate is not None:
            u = gate.astype(f32) * u
    if x is not None:
        s = f32(residual_scale) * x.astype(f32)
        u = s if u is None else s + u
    return u if wide else bf16_round(u)


def next_input(u, w_pre, eps):
    """bf16 rows (as float32) of the norm before a block, from the stream's float32 rows."""
    return bf16_round(u * inverse_rms(u, eps) * w_pre)


def joined(y_sorted, pair_offsets, pair_to_sorted, pair_weight, shared):
    """float64 rows of the experts' rows by their weights, and the sum of the terms' magnitudes."""
    T, d = len(pair_offsets) - 1, y_sorted.shape[1]
    y, ay = np.zeros((T, d)), np.zeros((T, d))
    for i in range(T):
        for p in range(pair_offsets[i], pair_offsets[i + 1]):
            t = float(pair_weight[p]) * y_sorted[pair_to_sorted[p]].astype(np.float64)
            y[i] += t
            ay[i] += np.abs(t)
    if shared is not None:
        y, ay = y + shared, ay + np.abs(shared)
    return y, ay
