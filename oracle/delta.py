"""Float64 CPU oracle of the gated delta rule and of the norms around its block: what ssm_delta_prefill,
ssm_delta_decode, ssm_gated_rmsnorm and ssm_block_rmsnorm compute, from their definitions, one token and head
at a time. Shares nothing with the library."""
from __future__ import annotations

import numpy as np


def softplus(x):
    return np.maximum(x, 0.0) + np.log1p(np.exp(-np.abs(x)))


def sigmoid(x):
    return 1.0 / (1.0 + np.exp(-x))


def gate(z, fn):
    return {"identity": lambda: z, "sigmoid": lambda: sigmoid(z), "silu": lambda: z * sigmoid(z), "tanh": lambda: np.tanh(z)}[fn]()


def split(qkv, hk, hv, dk, dv):
    x = np.asarray(qkv, np.float64)
    T = x.shape[0]
    return x[:, :hk * dk].reshape(T, hk, dk), x[:, hk * dk:2 * hk * dk].reshape(T, hk, dk), x[:, 2 * hk * dk:].reshape(T, hv, dv)


def step(S, q, k, v, alpha, beta):
    """One token of one head, S [dv][dk]: the new state and the output."""
    S = alpha * S
    S = S + np.outer(beta * (v - S @ k), k)
    return S, S @ q


def run(qkv, a, b, A_log, dt_bias, cu, slots, init, pool, hk, hv, dk, dv, qk_norm=True, scale=None, eps=1e-6, beta_max=1.0):
    """Packed sequences -> (o [T][hv][dv], the pool after the call, sizes [T][hv][dv]). sizes bounds what rounding
    errors are relative to: the absolute values of what is summed for an output, |S||q| summed over the state's row
    plus everything that decayed into it since the last multiple of 64 tokens."""
    q, k, v = split(qkv, hk, hv, dk, dv)
    scale = dk ** -0.5 if scale is None else scale
    pool = np.array(pool, np.float64)
    o, sizes = np.zeros(v.shape), np.zeros(v.shape)
    for i, slot in enumerate(slots):
        for h in range(hv):
            S = pool[slot, h].copy() if init[i] else np.zeros((dv, dk))
            mag = np.abs(S)
            for t in range(cu[i], cu[i + 1]):
                kt, qt = k[t, h // (hv // hk)], q[t, h // (hv // hk)]
                if qk_norm:
                    kt, qt = kt / np.sqrt(kt @ kt + eps), qt / np.sqrt(qt @ qt + eps)
                alpha = np.exp(-np.exp(A_log[h]) * softplus(a[t, h] + dt_bias[h]))
                beta = beta_max * sigmoid(b[t, h])
                if (t - cu[i]) % 64 == 0:
                    mag = np.abs(S)
                u = beta * (v[t, h] - alpha * S @ kt)
                mag = alpha * mag + np.outer(np.abs(u), np.abs(kt))
                S, y = step(S, qt * scale, kt, v[t, h], alpha, beta)
                o[t, h], sizes[t, h] = y, mag @ np.abs(qt * scale)
            pool[slot, h] = S
    return o, pool, sizes


def head_norm(x, w, z, eps, fn="silu", gate_first=False):
    """x [T][heads][dim]; w [dim] or [heads][dim]; z as x, or None."""
    f = 1.0 if z is None else gate(np.asarray(z, np.float64), fn)
    x = x * f if gate_first else x
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return y if gate_first else y * f


def block_norm(base, parts, norm_w, eps, post_w=None, post_eps=None, g=None, fn="identity", scale=1.0):
    y = sum([np.asarray(p, np.float64) for p in parts], np.zeros(base.shape))
    if post_w is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + (eps if post_eps is None else post_eps)) * post_w
    if g is not None:
        y = y * gate(np.asarray(g, np.float64), fn)
    r = base + scale * y
    return r, r / np.sqrt((r * r).mean(-1, keepdims=True) + eps) * norm_w
