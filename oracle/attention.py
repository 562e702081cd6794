"""Float64 CPU oracle of the paged attention cache: what ssm_kv_append, ssm_kv_read, ssm_attn_prefill and
ssm_attn_decode compute, from their definitions, one token and head at a time. Shares nothing with the
library."""
from __future__ import annotations

import numpy as np

CODE_MAX = {"fp8": 448.0, "int8": 127.0}
TINY = 1e-30


def round_e4m3(x):
    """float64 -> the nearest OCP E4M3 value (ties to even), |x| <= 448."""
    x = np.asarray(x, np.float64)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.abs(x)))
    step = 2.0 ** (np.maximum(np.where(np.isfinite(e), e, -6), -6) - 3)
    return np.round(x / step) * step


def decode_codes(codes, kind):
    """uint8 / int8 codes -> float64 values."""
    if kind == "int8":
        return np.asarray(codes).view(np.int8).astype(np.float64)
    c = np.asarray(codes).view(np.uint8).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (1 + m / 8.0) * 2.0 ** (e - 7.0), m / 8.0 * 2.0 ** -6)
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def quantise(x, kind):
    """[..., D] float64 -> (code values, scales)."""
    Q = CODE_MAX[kind]
    amax = np.abs(x).max(-1)
    amax = np.where(amax >= TINY, amax, 0.0)
    y = np.where(amax[..., None] > 0, x * (Q / np.where(amax > 0, amax, 1.0))[..., None], 0.0)
    return (round_e4m3(y) if kind == "fp8" else np.round(y)), amax / Q


def rms_norm(x, w, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def rotate(x, pos, radians, interleaved):
    """x [..., D] at one position; radians [rot / 2] per token."""
    h = len(radians)
    y = x.copy()
    for i, f in enumerate(radians):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        ang = float(np.fmod(np.longdouble(pos) * np.longdouble(f), np.longdouble("6.283185307179586476925286766559")))
        c, s = np.cos(ang), np.sin(ang)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def append(qkv, hq, hkv, pos, q_w, k_w, eps, radians, interleaved):
    """[T][(hq + 2 hkv) D] -> q [T][hq][D], k and v [T][hkv][D], before any rounding."""
    T = qkv.shape[0]
    x = np.asarray(qkv, np.float64).reshape(T, hq + 2 * hkv, -1)
    q, k, v = x[:, :hq].copy(), x[:, hq:hq + hkv].copy(), x[:, hq + hkv:].copy()
    if q_w is not None:
        q = rms_norm(q, q_w, eps)
    if k_w is not None:
        k = rms_norm(k, k_w, eps)
    for t in range(T):
        q[t] = rotate(q[t], pos[t], radians, interleaved)
        k[t] = rotate(k[t], pos[t], radians, interleaved)
    return q, k, v


def attend(q, k, v, positions, scale, window=0, ok=None):
    """q [m][hq][D] at `positions` over one sequence's k, v [n][hkv][D]; ok [n]: tokens that exist. Returns
    (o, sum of p |v|, largest |score| bound sum |q||k| scale): the latter two for error bounds."""
    m, hq, D = q.shape
    g = hq // k.shape[1]
    o, ab = np.zeros((m, hq, D)), np.zeros((m, hq, D))
    big = 0.0
    for t in range(m):
        p = int(positions[t])
        lo = max(0, p - window + 1) if window else 0
        idx = np.arange(lo, p + 1)
        if ok is not None:
            idx = idx[ok[lo:p + 1]]
        if idx.size == 0:
            continue
        for h in range(hq):
            kk, vv = k[idx, h // g], v[idx, h // g]
            s = kk @ q[t, h] * scale
            big = max(big, float((np.abs(kk) @ np.abs(q[t, h]) * scale).max()))
            e = np.exp(s - s.max())
            w = e / e.sum()
            o[t, h] = w @ vv
            ab[t, h] = w @ np.abs(vv)
    return o, ab, big
