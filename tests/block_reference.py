"""The operators around the layer in plain numpy, 64 bits: the norms with gate and residual scale, their gradients, and microscaled
4-bit numbers.  Written from the definitions in include/bigmac.h; nothing of the library's is used."""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24                        # half a step of fp32 at 1
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


# ------------------------------------------------------------------ norms

def statistics(v, kind, eps):
    m = v.mean(1, keepdims=True) if kind == "layer" else np.zeros((v.shape[0], 1))
    return m, 1.0 / np.sqrt(((v - m) ** 2).mean(1, keepdims=True) + eps)


def norm(v, w, b, kind, eps):
    m, r = statistics(v, kind, eps)
    n = (v - m) * r * w
    return n if b is None else n + b


def norm_gradient(v, w, c, kind, eps):
    """(gradient of v, of w, of b) for c, the gradient of norm(v, w, b)."""
    m, r = statistics(v, kind, eps)
    vh, a = (v - m) * r, c * w
    dv = a - vh * (a * vh).mean(1, keepdims=True)
    if kind == "layer":
        dv = dv - a.mean(1, keepdims=True)
    return dv * r, (c * vh).sum(0), c.sum(0)


def gate_values(g, gate, shape):
    if gate == "none":
        return np.ones(shape)
    return np.broadcast_to(g[:, None] if gate == "token" else g, shape).astype(np.float64)


def block_forward(x, y, p, kind, gate, eps, alpha):
    """z of the branch; p: post_w, post_b, gate."""
    return alpha * x + gate_values(p["gate"], gate, x.shape) * norm(y, p["post_w"], p["post_b"], kind, eps)


def block_backward(z, y, du, dz, p, kind, gate, eps, alpha):
    """Gradients of the whole call; y None: no branch; du None: no norm behind it."""
    out = {}
    dZ = np.zeros_like(z if z is not None else y) if dz is None else dz
    if du is not None:
        dv, out["d_pre_w"], out["d_pre_b"] = norm_gradient(z, p["pre_w"], du, kind, eps)
        dZ = dZ + dv
    out["dx"] = alpha * dZ
    if y is not None:
        g = gate_values(p["gate"], gate, y.shape)
        dg = dZ * norm(y, p["post_w"], p["post_b"], kind, eps)
        out["d_gate"] = {"none": lambda: None, "channel": lambda: dg.sum(0), "token": lambda: dg.sum(1), "full": lambda: dg}[gate]()
        out["dy"], out["d_post_w"], out["d_post_b"] = norm_gradient(y, p["post_w"], g * dZ, kind, eps)
    return out


# ------------------------------------------------------------------ 4-bit numbers

HELD = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(v):
    """(codes [.., n] 0..15, scale bytes [.., n / 32], values [.., n]) of rows in blocks of 32.  A block with an infinity or NaN: byte 255, codes 0, NaN."""
    v = np.asarray(v, np.float64)
    b = v.reshape(*v.shape[:-1], v.shape[-1] // 32, 32)
    top = np.abs(b).max(-1)
    finite = np.isfinite(top)
    power = np.frexp(np.where(finite, top, 1.0))[1] - 1                       # floor(log2 top)
    e = np.maximum(np.where(top > 0, power, -1000) - 2, -127)
    a = np.abs(np.where(finite[..., None], b, 0.0)) / np.exp2(e)[..., None]
    code = np.zeros(a.shape, np.int64)
    for c in range(1, 8):                                                     # past the middle between two neighbours, or on it towards the even code
        middle = 0.5 * (HELD[c - 1] + HELD[c])
        code[(a > middle) | ((a == middle) & (c % 2 == 0))] = c
    sign = np.signbit(b) & finite[..., None]
    values = np.where(sign, -1.0, 1.0) * HELD[code] * np.exp2(e)[..., None]
    values = np.where(finite[..., None], values, np.nan)
    return (code | (sign << 3)).reshape(v.shape), np.where(finite, e + 127, 255).astype(np.int64), values.reshape(v.shape)


def gelu(v):
    from scipy.special import erfc
    return 0.5 * v * erfc(-v / np.sqrt(2.0))


def ffn(x, counts, w1, w2, b1=None, b2=None):
    """The experts' FFN on 4-bit rows and held weights: (output, how far a bf16 result of the library may be off) per row.

    A product of n inputs adds 64 + n / 64 times in fp32, each off by at most a step of the partial sum (2 u), and once for the bias.  Where a hidden value
    lies within its own error of a border between two held values it may fall on either side: the output may be off by that step times the weight."""
    outs, limits, at = [], [], 0
    xq = quantise(x)[2]
    for e, n in enumerate(counts):
        a = xq[at:at + n]
        pre, size = a @ w1[e], np.abs(a) @ np.abs(w1[e])
        if b1 is not None:
            pre, size = pre + b1[e], size + np.abs(b1[e])
        h = gelu(pre)
        # |gelu'| < 1.13; the library's GELU: a polynomial within 6.8e-7 of gelu (of |a| times it below 1), its exponential within a step, 1.2e-7
        # of at most half of |a|
        off = 1.13 * 2 * (65 + a.shape[1] / 64) * U32 * size + 8e-7 + 4 * U32 * np.abs(h)
        q = quantise(h)[2]
        moved = np.zeros_like(q)
        for direction in (1.0, -1.0):                                # all magnitudes a little larger, a little smaller: also across a scale's border
            there = quantise(np.where(h < 0, -1.0, 1.0) * np.maximum(np.abs(h) + direction * off, 0.0))[2]
            moved = np.maximum(moved, np.abs(there - q))
        want, osize = q @ w2[e], np.abs(q) @ np.abs(w2[e])
        if b2 is not None:
            want, osize = want + b2[e], osize + np.abs(b2[e])
        outs.append(want)
        limits.append(2 * (65 + h.shape[1] / 64) * U32 * osize + HALF_STEP["bf16"] * np.abs(want) * (1 + 2.0 ** -10) + (1 + HALF_STEP["bf16"]) * (moved @ np.abs(w2[e])))
        at += n
    return np.concatenate(outs), np.concatenate(limits)
