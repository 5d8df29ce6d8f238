"""Plain forms of a step's work for each token in 64 bits (numpy), with the bounds of what 32-bit sums and one rounding of
the output may be off."""

import math

import numpy as np

U = {"bf16": 2.0**-8, "f16": 2.0**-11}      # half a step relative to the value
TINY = {"bf16": 2.0**-126, "f16": 2.0**-24}  # what a value below the normal range may lose (f16: a step; bf16: fp32's own least)

_erf = np.vectorize(math.erf, otypes=[float])
_erfc = np.vectorize(math.erfc, otypes=[float])


def act(v, name):
    with np.errstate(over="ignore", invalid="ignore"):
        if name == "silu":
            return v / (1 + np.exp(-v))
        if name == "gelu":
            return 0.5 * v * _erfc(-v / math.sqrt(2))
        if name == "gelu_tanh":
            return v / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v**3)))
        return np.where(v < 0, 0.0, v) if name == "relu" else v


def product(x, w, bias):
    """x w^T + bias, and how far the same in fp32 may be from it: K products summed with each partial sum cut rather than
    rounded (2^-22 of the sum of magnitudes each), then the bias."""
    with np.errstate(invalid="ignore"):
        v, size = x @ w.T, np.abs(x) @ np.abs(w).T
        if bias is not None:
            v, size = v + bias, size + np.abs(bias)
        return v, (x.shape[1] + 1) * 2.0**-22 * size


def linear(x, w, bias, name, residual, dtype):
    """lv_linear and its bound.  No activation's slope is above 1.13; its own arithmetic (an exponential of an argument
    that is good to 2^-23 of it, a sum, a quotient: 2^-16 where the result is not below 2^-126) is relative to its value."""
    v, dv = product(x, w, bias)
    y = act(v, name)
    dy = (1.0 if name in ("none", "relu") else 1.13) * dv + (0 if name in ("none", "relu") else 2.0**-16) * np.abs(y)
    if residual is not None:
        y = y + residual
        dy = dy + 2.0**-23 * (np.abs(y) + np.abs(residual))
    return y, dy + U[dtype] * (np.abs(y) + dy) + TINY[dtype]


def gated(x, wg, wu, bg, bu, name, dtype):
    """lv_gated_linear and its bound."""
    g, dg = product(x, wg, bg)
    u, du = product(x, wu, bu)
    a = act(g, name)
    da = (1.0 if name in ("none", "relu") else 1.13) * dg + (0 if name in ("none", "relu") else 2.0**-16) * np.abs(a) + 2.0**-126
    y = a * u
    dy = da * np.abs(u) + np.abs(a) * du + da * du + 2.0**-23 * np.abs(y)
    return y, dy + U[dtype] * (np.abs(y) + dy) + TINY[dtype]


def positions(n_tok, offsets, c):
    """The position of every token, -1 for tokens of no request."""
    pos = np.full(n_tok, -1, np.int64)
    for i in range(len(offsets) - 1):
        for t in range(offsets[i], offsets[i + 1]):
            pos[t] = t - offsets[i] + (0 if c is None else c[i])
    return pos


def rotate(x, weight, eps, pos, freq, neighbours, dtype):
    """lv_qk_rotate of one array [n_tok][heads][d], and its bound: the norm's sum of d squares, its root and quotient, the
    weight and two products and a sum of the rotation, each good to 2^-23 or better; cos and sin good to 2^-22 absolute
    (the angle's remainder, in [-pi, pi], is rounded to 24 bits: pi 2^-24, and the functions add 2^-23) and to what 64 bits
    leave of the angle."""
    x = x.astype(np.float64)
    d, half = x.shape[-1], len(freq)
    if weight is not None:
        with np.errstate(invalid="ignore", divide="ignore"):
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    y = x.copy()
    dy = (d * 2.0**-23 if weight is not None else 0) * np.abs(x)
    if half:
        j = np.arange(half)
        a, b = (2 * j, 2 * j + 1) if neighbours else (j, j + half)
        angle = pos[:, None].astype(np.float64) * np.asarray(freq)
        da = (2.0**-22 + 2.0**-51 * np.abs(angle))[:, None, :]
        co, si = np.cos(angle)[:, None, :], np.sin(angle)[:, None, :]
        size = np.abs(x[..., a]) + np.abs(x[..., b])
        y[..., a] = x[..., a] * co - x[..., b] * si
        y[..., b] = x[..., a] * si + x[..., b] * co
        off = (2.0**-22 + da + (d * 2.0**-23 if weight is not None else 0)) * size
        dy[..., a] = off
        dy[..., b] = off
    return y, dy + U[dtype] * (np.abs(y) + dy) + TINY[dtype]


def logprobs(x, ids, n_top):
    """lv_token_logprobs row by row: logp, entropy, lse, top ids, top log probabilities.  A difference of two logits may be
    beyond fp32's range, which its outputs hold as an infinity."""
    n, V = x.shape
    logp, ent, lse = np.full(n, np.nan), np.full(n, np.nan), np.full(n, np.nan)
    top_ids, top_lp = np.full((n, n_top), -1, np.int64), np.full((n, n_top), -np.inf)
    for t in range(n):
        v = x[t].astype(np.float64)
        k = min(n_top, V)
        order = np.lexsort((np.arange(V), -np.where(np.isnan(v), 0, v), ~np.isnan(v)))[:k]
        top_ids[t, :k] = order
        nan = np.isnan(v).any()
        m = v.max()
        with np.errstate(invalid="ignore"):
            if nan:
                lse[t], lp = np.nan, np.full(V, np.nan)
            elif m == -np.inf:
                lse[t], ent[t], lp = -np.inf, 0.0, np.full(V, -np.inf)
            elif m == np.inf:
                lse[t], lp = np.inf, v - np.inf
            else:
                e = np.exp(v - m)
                S = e.sum()
                lse[t] = m + np.log(S)
                lp = v - m - np.log(S)
                with np.errstate(divide="ignore"):
                    ent[t] = np.log(S) - np.where(e > 0, e * np.where(e > 0, v - m, 0), 0).sum() / S
        lp = np.where(lp < -float(np.finfo(np.float32).max), -np.inf, lp)
        if 0 <= ids[t] < V:
            logp[t] = lp[ids[t]]
        top_lp[t, :k] = lp[order]
    return logp, ent, lse, top_ids, top_lp
