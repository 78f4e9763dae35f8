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
