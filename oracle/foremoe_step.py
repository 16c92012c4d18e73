"""Oracle of the operators around the expert layer: the router, the
log-probabilities of given tokens and the AdamW step, in numpy float64 from
their definitions (include/foremoe.h). The 8-bit optimizer states are defined
by fp32 operations one after another, so adamw8_step does those in float32.
"""
from __future__ import annotations

import numpy as np

INF = np.inf


# ---------------------------------------------------------------------------
# Router (Sec. 2.1; replayed ids, Sec. 5)
# ---------------------------------------------------------------------------
def _scores(l, score):
    """(s, pi) of one row: its scores and their distribution."""
    with np.errstate(over="ignore", invalid="ignore", under="ignore"):
        if score == "sigmoid":
            s = 1.0 / (1.0 + np.exp(-l))
            total = s.sum()
            return s, s / total if total != 0 else np.zeros_like(s)
        top = np.max(np.where(np.isnan(l), -INF, l))
        e = np.exp(l - (0.0 if top == -INF else top))
        return e / e.sum(), e / e.sum()


def router_pick(l, K, bias=None):
    """The K places of one row of logits: ids, -1 where left over."""
    l = np.asarray(l, dtype=np.float64)
    key = l if bias is None else _scores(l, "sigmoid")[0] + bias
    key = np.where((l > -INF) & (key > -INF), key, -INF)  # False for a NaN
    order = sorted(range(len(l)), key=lambda e: (-key[e], e))[:K]
    return np.array([e if key[e] > -INF else -1 for e in order], dtype=np.int32)


def _gates(l, ids, score, renorm, scale):
    """One row's (gates, d gates / d logits [K, E])."""
    E, K = len(l), len(ids)
    s, _ = _scores(l, score)
    there = ids >= 0
    picked = np.where(there, s[np.maximum(ids, 0)], 0.0)
    # d s_k / d l_e
    ds = np.zeros((K, E))
    for k in np.nonzero(there)[0]:
        if score == "sigmoid":
            ds[k, ids[k]] = picked[k] * (1 - picked[k])
        else:
            ds[k] = -picked[k] * s
            ds[k, ids[k]] += picked[k]
    if renorm:
        if score == "softmax" and there.any():  # the sum of the scores cancels
            x = np.where(there, l[np.maximum(ids, 0)], -INF)
            top = np.max(np.where(np.isnan(x), -INF, x))
            with np.errstate(invalid="ignore"):
                picked = np.where(there, np.exp(x - (0.0 if top == -INF else top)), 0.0)
            ds = np.zeros((K, E))
            for k in np.nonzero(there)[0]:
                ds[k, ids[k]] = picked[k]
        total = picked.sum()
        if total == 0:
            return np.zeros(K), np.zeros((K, E))
        q = picked / total
        return scale * q, scale * (ds - q[:, None] * ds.sum(0)[None, :]) / total
    return scale * picked, scale * ds


def router_forward(logits, K, *, score="softmax", renorm=True, scale=1.0, bias=None, mask=None, ids=None):
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    out_ids = np.full((T, K), -1, dtype=np.int32)
    gates = np.zeros((T, K))
    psum, n = np.zeros(E), 0
    for t in range(T):
        l = logits[t]
        if (mask is not None and not mask[t]) or np.all(l == -INF):
            continue
        if ids is None:
            i = router_pick(l, K, bias)
        else:
            i = np.array(ids[t], dtype=np.int32)
            i[(i < 0) | (i >= E)] = -1
            i[(i >= 0) & (l[np.maximum(i, 0)] == -INF)] = -1
        out_ids[t] = i
        gates[t] = _gates(l, i, score, renorm, scale)[0]
        psum += _scores(l, score)[1]
        n += 1
    counts = np.bincount(out_ids[out_ids >= 0], minlength=E).astype(np.int32)
    mean = psum / max(n, 1)
    loss = E * np.sum(counts / max(1, counts.sum()) * mean)
    return dict(ids=out_ids, gates=gates, counts=counts, n_tokens=n, prob_mean=mean, balance_loss=loss)


def router_backward(logits, ids, dgates, *, score="softmax", renorm=True, scale=1.0, mask=None, counts=None,
                    n_tokens=None, balance_coef=0.0):
    logits = np.asarray(logits, dtype=np.float64)
    T, E = logits.shape
    out = np.zeros((T, E))
    for t in range(T):
        l = logits[t]
        if (mask is not None and not mask[t]) or np.all(l == -INF):
            continue
        if dgates is not None:
            i = np.where((ids[t] >= 0) & (ids[t] < E), ids[t], -1)
            dg = np.where(i >= 0, dgates[t], 0.0)
            out[t] += dg @ _gates(l, i, score, renorm, scale)[1]
        if balance_coef != 0:
            s, pi = _scores(l, score)
            c = balance_coef * E / max(n_tokens, 1) * counts / max(1, counts.sum())
            r = pi * (c - pi @ c)
            out[t] += r * (1 - s) if score == "sigmoid" else r
    return out


# ---------------------------------------------------------------------------
# Log-probabilities of given tokens
# ---------------------------------------------------------------------------
def _xlogx(p, lp):
    with np.errstate(invalid="ignore"):
        return np.where(p > 0, p * lp, p * 0)  # keeps a NaN


def token_logprobs(logits, targets=None, *, temperature=1.0, n_top=0):
    logits = np.asarray(logits, dtype=np.float64)
    N, V = logits.shape
    r = dict(logp=np.zeros(N), entropy=np.zeros(N), lse=np.zeros(N), top_ids=np.full((N, n_top), -1, dtype=np.int32),
             top_logp=np.full((N, n_top), -INF))
    for i in range(N):
        if targets is not None and not 0 <= targets[i] < V:
            continue
        x = logits[i] / temperature
        top = np.max(np.where(np.isnan(x), -INF, x))
        none = np.all(x == -INF)
        with np.errstate(invalid="ignore", divide="ignore"):
            top = 0.0 if top == -INF else top
            d = x - top  # the largest first, so that log-probabilities of huge logits keep their digits
            ls = np.log(np.sum(np.exp(d)))
            lse, lp = top + ls, d - ls
        r["lse"][i] = lse
        r["entropy"][i] = 0.0 if none else -np.sum(_xlogx(np.exp(lp), lp))
        if targets is not None:
            r["logp"][i] = -INF if none else lp[targets[i]]
        order = np.lexsort((np.arange(V), -np.where(np.isnan(x), -INF, logits[i])))[:n_top]
        for k, j in enumerate(order):
            if x[j] > -INF:
                r["top_ids"][i, k], r["top_logp"][i, k] = j, lp[j]
    return r


def token_logprobs_backward(logits, targets, dlogp=None, dentropy=None, *, temperature=1.0):
    logits = np.asarray(logits, dtype=np.float64)
    N, V = logits.shape
    f = token_logprobs(logits, targets, temperature=temperature)
    out = np.zeros((N, V))
    for i in range(N):
        if targets is not None and not 0 <= targets[i] < V:
            continue
        with np.errstate(invalid="ignore"):
            lp = logits[i] / temperature - f["lse"][i]
        p = np.zeros(V) if f["lse"][i] == -INF else np.exp(lp)
        if dlogp is not None:
            out[i] -= dlogp[i] * p
            out[i, targets[i]] += dlogp[i]
        if dentropy is not None:
            out[i] -= dentropy[i] * (_xlogx(p, lp) + p * f["entropy"][i])
    return out / temperature


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
BLOCK = 256


def adamw_step(p, g, m, v, *, lr, beta1, beta2, eps, weight_decay, step, grad_scale=1.0):
    """(p, m, v) after one step, float64."""
    p, g, m, v = (np.asarray(a, dtype=np.float64) for a in (p, g, m, v))
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mh, vh = m / (1 - beta1 ** step), v / (1 - beta2 ** step)
    return p * (1 - lr * weight_decay) - lr * mh / (np.sqrt(vh) + eps), m, v


def code_table(fraction_bits, codes):
    """The value over its scale of every code: code 0 is 0, the last one 1,
    each octave below holds 2^fraction_bits evenly spaced values."""
    out = np.zeros(codes)
    per = 1 << fraction_bits
    for c in range(1, codes):
        k = c - (codes - 1)  # 0 at 1.0
        e = k // per
        out[c] = 2.0 ** e * (1 + (k - e * per) / per)
    return out


TABLE_M, TABLE_V = code_table(3, 128), code_table(4, 256)


def _nearest(x, table):
    """The code whose value is nearest to x, in the middle the one with an
    even last bit of its float pattern (codes and patterns differ by an odd
    number, so an odd code)."""
    hi = np.clip(np.searchsorted(table[1:], x) + 1, 1, len(table) - 1)
    lo = hi - 1
    up, dn = table[hi] - x, x - table[lo]
    tie = np.where(hi % 2 == 1, hi, lo)
    c = np.where(up < dn, hi, np.where(dn < up, lo, tie))
    return c


def _blocks(a):
    n = a.size
    out = np.zeros(-(-n // BLOCK) * BLOCK, dtype=a.dtype)
    out[:n] = a.reshape(-1)
    return out.reshape(-1, BLOCK)


def _inverse(scale):
    one = np.float32(1)
    tiny = np.float32(2.0 ** -126)
    return np.where(scale >= tiny, one / np.where(scale >= tiny, scale, one), np.float32(0))


def encode_m(m):
    """(codes uint8 [n], scales fp32) of fp32 first moments."""
    a = _blocks(np.abs(m.astype(np.float32)))
    scale = a.max(1)
    x = (a * _inverse(scale)[:, None]).astype(np.float32).astype(np.float64)
    c = _nearest(np.minimum(x, 1.0), TABLE_M)
    # below the smallest code by half a step of its own octave: 0
    c = np.where(x < _least(3, 127), 0, np.maximum(c, 1))
    c = np.where((_blocks(m) < 0) & (c > 0), c + 128, c)
    return c.reshape(-1)[:m.size].astype(np.uint8), scale


def encode_v(v):
    u = np.sqrt(_blocks(v.astype(np.float32)))
    scale = u.max(1)
    x = (u * _inverse(scale)[:, None]).astype(np.float32).astype(np.float64)
    c = np.maximum(_nearest(np.minimum(x, 1.0), TABLE_V), 1)
    c = np.where(x > 0, c, 0)
    return c.reshape(-1)[:v.size].astype(np.uint8), scale


def _least(fraction_bits, top):
    """What rounds up to code 1 (the pattern below it, code 0's place, would
    hold the value one step under code 1; the middle has an odd last bit
    above it)."""
    per = 1 << fraction_bits
    value = lambda k: 2.0 ** (k // per) * (1 + (k % per) / per)  # noqa: E731
    return (value(-top) + value(1 - top)) / 2


def decode_m(c, scale):
    x = (TABLE_M.astype(np.float32)[c & 127].reshape(-1))
    s = np.repeat(scale, BLOCK)[:c.size]
    x = (x * s).astype(np.float32)
    return np.where(c >= 128, -x, x).astype(np.float32)


def decode_v(c, scale):
    u = (TABLE_V.astype(np.float32)[c] * np.repeat(scale, BLOCK)[:c.size]).astype(np.float32)
    return (u * u).astype(np.float32)


def adamw8_moments(g, cm, sm, cv, sv, *, beta1, beta2, grad_scale=None):
    """fp32 moments (m, v) of one step on 8-bit states, each operation rounded
    to fp32, and the new states (codes and scales)."""
    f = np.float32
    g = g.astype(f)
    if grad_scale is not None:
        g = g * f(grad_scale)
    m = decode_m(cm, sm) * f(beta1) + g * f(1 - beta1)
    v = decode_v(cv, sv) * f(beta2) + (g * g) * f(1 - beta2)
    return m, v, encode_m(m), encode_v(v)
