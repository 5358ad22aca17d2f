"""Test infrastructure: plain 64-bit definitions of the calls on tokens (numpy), sharing no code with the library."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def rotate(x, weight, pos, sections, base, pairs="split", ladder="axis", eps=1e-6):
    """x [tokens][heads][dim] -> float64; weight [dim] or None; pos [tokens][axes]."""
    u = np.asarray(x, np.float64).copy()
    if weight is not None:
        u = u / np.sqrt((u * u).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    y, total, p = u.copy(), sum(sections), 0
    for a, count in enumerate(sections):
        for j in range(count):
            f = float(base) ** (-(j / count if ladder == "axis" else p / total))
            ang = pos[:, a].astype(np.float64) * f
            c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
            i, k = (p, p + total) if pairs == "split" else (2 * p, 2 * p + 1)
            y[..., i] = u[..., i] * c - u[..., k] * s
            y[..., k] = u[..., k] * c + u[..., i] * s
            p += 1
    return y


def mx4_encode(x, cap=252):
    """(codes as 0..15 per value, exponent bytes per group of 32) of float64 [..., n]."""
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (-1, 32))
    most = np.abs(g).max(-1)
    e = np.full(most.shape, -126, np.int64)
    while True:
        more = np.isfinite(g).all(-1) & (e < cap - 127) & (most > 7.0 * np.exp2(e.astype(np.float64)))
        if not more.any():
            break
        e[more] += 1
    finite = np.isfinite(g).all(-1)
    q = np.abs(np.where(finite[..., None], g, 0.0)) / np.exp2(e.astype(np.float64))[..., None]
    mids = (E2M1[1:] + E2M1[:-1]) / 2
    low, high = np.searchsorted(mids, q, "left"), np.searchsorted(mids, q, "right")     # differ only on a tie
    code = np.where(low % 2 == 0, low, high)
    code = code | np.where(np.signbit(g), 8, 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(finite, e + 127, 255).astype(np.uint8)


def mx4_decode(codes, exps):
    """float64 values of codes [..., n] with exponent bytes [..., n / 32]."""
    v = E2M1[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(exps == 255, np.nan, np.exp2(exps.astype(np.float64) - 127.0))
    return v * np.repeat(s, 32, -1)


def mx4_pack(codes):
    """Two codes a byte, the even index in the low half."""
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def mx4_unpack(b):
    out = np.empty(b.shape[:-1] + (2 * b.shape[-1],), np.uint8)
    out[..., 0::2], out[..., 1::2] = b & 15, b >> 4
    return out


def attend(q, k, v, q_start, kv_start, kv_len, scale, key_mask=None):
    """(out, lse) in float64.  q [n_q][Hq][D], k and v [rows][Hk][D]; sequence b owns queries q_start[b] .. q_start[b + 1] and the
    keys kv_start[b] .. + kv_len[b]; rows of no sequence stay NaN."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    n_q, hq, _ = q.shape
    group = hq // k.shape[1]
    out, lse = np.full(q.shape[:2] + (v.shape[2],), np.nan), np.full((n_q, hq), np.nan)
    for b in range(len(kv_start)):
        lo, hi = int(q_start[b]), int(q_start[b + 1])
        rows = np.arange(int(kv_start[b]), int(kv_start[b]) + int(kv_len[b]))
        see = rows if key_mask is None else rows[np.asarray(key_mask)[rows] != 0]
        for h in range(hq):
            if not len(see):
                out[lo:hi, h], lse[lo:hi, h] = 0.0, -np.inf
                continue
            with np.errstate(invalid="ignore"):
                s = q[lo:hi, h] @ k[see, h // group].T * scale
                top = s.max(-1, keepdims=True)
                p = np.exp(s - top)
                out[lo:hi, h], lse[lo:hi, h] = p @ v[see, h // group] / p.sum(-1, keepdims=True), top[:, 0] + np.log(p.sum(-1))
    return out, lse
