"""Test infrastructure: plain 64-bit definitions of the calls around attention (numpy), sharing no code with the library."""
from __future__ import annotations

import math

import numpy as np

from .fp8 import e4m3_decode


def mx8_encode(x):
    """(E4M3 codes, exponent bytes per group of 32) of float64 [..., n]."""
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, 32))
    finite = np.isfinite(g).all(-1)
    g = np.where(finite[..., None], g, 0.0)
    most = np.abs(g).max(-1)
    e = np.full(most.shape, -126, np.int64)
    while True:
        more = most > 448.0 * np.exp2(e.astype(np.float64))
        if not more.any():
            break
        e[more] += 1
    values = e4m3_decode(np.arange(127, dtype=np.uint8))       # 0 .. 448, ascending with the code
    mids = (values[1:] + values[:-1]) / 2
    q = np.abs(g) / np.exp2(e.astype(np.float64))[..., None]
    low, high = np.searchsorted(mids, q, "left"), np.searchsorted(mids, q, "right")     # differ only on a tie
    code = np.where(low % 2 == 0, low, high) | np.where(np.signbit(g), 128, 0)
    code = np.where(finite[..., None], code, 0x7F)
    return code.reshape(x.shape).astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def mx8_decode(codes, exps):
    """float64 values of codes [..., n] with exponent bytes [..., n / 32]."""
    s = np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127.0))
    return e4m3_decode(codes) * np.repeat(s, 32, -1)


def norm(x, res=None, weight=None, eps=1e-6, norm=True):
    """(s, y) in float64."""
    s = np.asarray(x, np.float64) if res is None else np.asarray(x, np.float64) + np.asarray(res, np.float64)
    y = s
    if norm:
        with np.errstate(invalid="ignore", over="ignore"):
            y = s / np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    return s, y if weight is None else y * np.asarray(weight, np.float64)


_erf = np.vectorize(math.erf)


def activate(name, v):
    with np.errstate(over="ignore"):
        return {"none": lambda: v, "relu": lambda: np.maximum(v, 0.0), "silu": lambda: v / (1.0 + np.exp(-v)), "gelu": lambda: 0.5 * v * (1.0 + _erf(v * math.sqrt(0.5)))}[name]()


def product(x, w, bias=None, act="none", gated=False, res=None):
    """act(x w^T + bias) in float64; gated: the first half of w's rows, activated, times the second; then + res."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    half = z.shape[1] // 2
    y = activate(act, z[:, :half]) * z[:, half:] if gated else activate(act, z)
    return y if res is None else y + np.asarray(res, np.float64)


def kept_tokens(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """The tokens of a row of logits that may be drawn, best first, and their weights (the best one's is 1)."""
    x = np.asarray(x, np.float64)
    words = [i for i in range(len(x)) if x[i] > -np.inf]
    words.sort(key=lambda i: (-x[i], i))
    if not words:
        return [], []
    greedy = not temperature > 0
    top = x[words[0]]
    weight = [1.0 if greedy or x[i] == top else 0.0 if np.isinf(top) else math.exp((x[i] - top) / temperature) for i in words]
    count = 1 if greedy else min(top_k, len(words)) if top_k > 0 else len(words)
    total = math.fsum(weight[:count])
    keep, before = 0, []
    for r in range(count):
        if r and (top_p < 1 and math.fsum(before) >= top_p * total or weight[r] < min_p):
            break
        before.append(weight[r])
        keep += 1
    return words[:keep], weight[:keep]


def sample(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, number of tokens it was drawn from, log of its probability among them); -1, 0, -inf where no token is left."""
    words, weight = kept_tokens(x, temperature, top_k, top_p, min_p)
    if not words:
        return -1, 0, -np.inf
    total = math.fsum(weight)
    by_index = sorted(zip(words, weight))
    up_to = 0.0
    for i, w in by_index:
        up_to += w
        if w and up_to > u * total:
            return i, len(words), math.log(w / total)
    i, w = [p for p in by_index if p[1]][-1]
    return i, len(words), math.log(w / total)
