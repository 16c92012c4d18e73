"""Oracle of the operators that take the experts' weights from an update to the
rollout: microscaled 4-bit floats, the expert FFN in them, the expert layer for
a few tokens and the Muon step, in numpy float64 from their definitions
(include/foremoe.h).
"""
from __future__ import annotations

import numpy as np

MX = 32
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NAN_SCALE = 255


# ---------------------------------------------------------------------------
# Microscaled 4-bit floats
# ---------------------------------------------------------------------------
def mx_exponent(amax):
    """The least e with amax < 7 * 2^e, within [-127, 125]."""
    amax = np.asarray(amax, dtype=np.float64)
    e = np.full(amax.shape, -127)
    # compared with exact products, exponent by exponent
    for k in range(-127, 125):
        e = np.where(amax >= 7 * 2.0 ** k, k + 1, e)
    return e


def mx_round(y):
    """(place in GRID, sign) of the nearest of +-GRID, ties to the even place."""
    a = np.abs(np.asarray(y, dtype=np.float64))
    dist = np.abs(a[..., None] - GRID)
    near = dist == dist.min(-1, keepdims=True)
    # of two equally near places the even one
    place = np.where(near, np.arange(8), 99).min(-1)
    other = np.where(near, np.arange(8), -1).max(-1)
    place = np.where((place != other) & (place % 2 == 1), other, place)
    return place, np.signbit(y)


def mxfp4_quantize(x):
    """codes [..., 16 * blocks] and scales [..., blocks] (uint8) of x [..., n]."""
    x = np.asarray(x, dtype=np.float64)
    n = x.shape[-1]
    pad = -n % MX
    b = np.concatenate([x, np.zeros((*x.shape[:-1], pad))], -1).reshape(*x.shape[:-1], -1, MX)
    bad = ~np.isfinite(b).all(-1)
    b = np.where(bad[..., None], 0.0, b)
    e = mx_exponent(np.abs(b).max(-1))
    place, sign = mx_round(b / 2.0 ** e[..., None])
    code = (place + 8 * sign).astype(np.uint8)
    code = np.where(bad[..., None], 0, code).astype(np.uint8).reshape(*x.shape[:-1], -1)
    scales = np.where(bad, NAN_SCALE, e + 127).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, scales


def mxfp4_values(codes, scales, n=None):
    c = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)
    v = np.where(c >= 8, -1.0, 1.0) * GRID[c & 7]
    s = np.where(scales == NAN_SCALE, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    v = (v.reshape(*scales.shape, MX) * s[..., None]).reshape(*codes.shape[:-1], -1)
    return v if n is None else v[..., :n]


def silu(a):
    with np.errstate(over="ignore"):
        return a / (1.0 + np.exp(-a))


def ffn_mxfp4(x, gate_up, down):
    """One slot's rows. x [n, d], gate_up [2F, d], down [d, F]: the values that
    the codes stand for. Returns (h before it is quantised, y)."""
    F = down.shape[1]
    a, u = x @ gate_up[:F].T, x @ gate_up[F:].T
    h = silu(a) * u
    return h, mxfp4_values(*mxfp4_quantize(h), F) @ down.T


# ---------------------------------------------------------------------------
# The layer for a few tokens
# ---------------------------------------------------------------------------
def few_tokens(x, ids, gates, gate_up, down, expert_widx=None):
    """y [T, d]; gate_up [W, 2F, d], down [W, d, F]."""
    W, d, F = down.shape
    y = np.zeros((x.shape[0], d))
    E = W if expert_widx is None else len(expert_widx)
    for t in range(x.shape[0]):
        for k in range(ids.shape[1]):
            e = ids[t, k]
            if not 0 <= e < E:
                continue
            w = e if expert_widx is None else expert_widx[e]
            if not 0 <= w < W:
                continue
            g = gate_up[w] @ x[t]
            y[t] += gates[t, k] * (down[w] @ (silu(g[:F]) * g[F:]))
    return y


# ---------------------------------------------------------------------------
# Muon
# ---------------------------------------------------------------------------
def newton_schulz(x, coef, steps):
    """steps of X = a X + (b G + c G G) X, G = X X^T, on the smaller side."""
    a, b, c = coef
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for _ in range(steps):
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if tall else x


def newton_schulz_held(x, coef, steps):
    """The same with the roundings that the step's format has, or coarser ones. A
    side of at most 64: G and the product of all M = a I + b G + c G G in fp32, X =
    Q X0 (the step has fp64 there, and forms G again after some steps). Else
    the products' factors in fp16, of X the first of two numbers; the last step
    does without the second (unless it is the first too)."""
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    if min(x.shape) <= 64:
        f = np.float32
        a, b, c = (f(v) for v in coef)
        g = x.astype(f) @ x.astype(f).T
        q = np.eye(len(x), dtype=f)
        for _ in range(steps):
            m = a * np.eye(len(x), dtype=f) + b * g + c * (g @ g)
            q = m @ q
            g = m @ g @ m
        x = (q @ x.astype(f)).astype(np.float64)
        return x.T if tall else x
    a, b, c = coef
    half = lambda v: v.astype(np.float16).astype(np.float64)  # noqa: E731
    x = x * 256
    for i in range(steps):
        hi = half(x)
        x = hi + half((x - hi) * 1024) / 1024 if i == 0 or i + 1 < steps else hi
        g = half(hi @ hi.T / 256)
        p = half(b * g + c * (g @ g) / 256)
        x = a * x + p @ hi / 256
    x = x / 256
    return x.T if tall else x


def muon_step(p, grad, m, *, lr, momentum, nesterov, steps, coef, eps, weight_decay, scale, grad_scale=1.0,
              iterate=newton_schulz):
    """One matrix: (p, m, X) after the step."""
    g = grad * grad_scale
    m = momentum * m + g
    u = g + momentum * m if nesterov else m
    norm = np.sqrt((u * u).sum())
    den = max(norm, eps)
    x = iterate(u / den, coef, steps) if den > 0 else np.zeros_like(u)
    return p * (1 - lr * weight_decay) - lr * scale * x, m, x
