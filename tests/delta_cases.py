"""Shared by the tests of the gated delta rule: a layer's inputs on the host, their copies on the GPU, and the bounds
that the outputs are held to."""
import numpy as np

from oracle import delta as od


class Layer:
    """qkv, b and a of sequences of the given lengths; everything representable in the activation type. The projection's
    columns are z | b | a, and its rows end in columns of another user."""

    def __init__(self, torch, heads, lens, act, seed=0, spare=2, init=None, qk_norm=True, beta_max=1.0, decay=None):
        rng = np.random.default_rng(seed)
        self.torch, self.heads, self.lens, self.act = torch, heads, list(lens), act
        self.hk, self.hv, self.dk, self.dv = heads
        self.qk_norm, self.beta_max = qk_norm, beta_max
        hk, hv, dk, dv = heads
        n, T = len(lens), sum(lens)
        self.T, self.n, self.S = T, n, n + spare
        self.tdt = torch.bfloat16 if act == "bf16" else torch.float32
        x = rng.standard_normal((T, 2 * hk * dk + hv * dv))
        x = x * od.sigmoid(x)
        if not qk_norm:
            qk = x[:, :2 * hk * dk].reshape(T, 2 * hk, dk)
            x[:, :2 * hk * dk] = (qk / np.sqrt((qk * qk).sum(-1, keepdims=True) + 1e-6)).reshape(T, -1)
        self.qkv = self.stored(x)
        self.wide = hv * dv
        self.proj = self.stored(rng.standard_normal((T, -(-(self.wide + 2 * hv) // 8) * 8 + 8)))
        self.A_log = np.log(rng.uniform(1, 16, hv)).astype(np.float32)
        dt = np.exp(rng.uniform(np.log(1e-3), np.log(0.1), hv))
        self.dt_bias = (dt + np.log(-np.expm1(-dt))).astype(np.float32)
        if decay is not None:   # log decay per token of about -decay
            self.A_log[:], self.dt_bias[:] = np.log(decay), np.log(np.expm1(1.0))
        self.cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.slots = rng.permutation(self.S)[:n].astype(np.int32)
        self.init = (rng.random(n) < 0.5).astype(np.int32) if init is None else np.array(init, np.int32)
        self.pool = (0.3 * rng.standard_normal((self.S, hv, dv, dk))).astype(np.float32)

    def stored(self, x):
        """x rounded to the activation type, as float32."""
        t = self.torch.from_numpy(np.ascontiguousarray(x, np.float32))
        return t.to(self.tdt).float().numpy()

    def columns(self, x):
        """z, b and a of the projection."""
        w, hv = self.wide, self.hv
        return x[:, :w], x[:, w:w + hv], x[:, w + hv:w + 2 * hv]

    def oracle(self, pool=None, init=None):
        _, b, a = self.columns(self.proj.astype(np.float64))
        return od.run(self.qkv, a, b, self.A_log.astype(np.float64), self.dt_bias.astype(np.float64), self.cu, self.slots,
                      self.init if init is None else init, self.pool if pool is None else pool, *self.heads,
                      qk_norm=self.qk_norm, beta_max=self.beta_max)

    def dev(self, x, act=True):
        t = self.torch.from_numpy(np.ascontiguousarray(x))
        return t.to(self.tdt if act else t.dtype).cuda()

    def desc(self, B):
        return B.make_delta_desc(*self.heads, act=self.act, qk_norm=self.qk_norm, beta_max=self.beta_max)

    def gates(self, B, dd):
        return B.DeltaGates(dd, self.dev(self.A_log, False), self.dev(self.dt_bias, False))


def f64(t):
    return t.detach().to("cpu").double().numpy()


def out_bound(want, sizes, act):
    """Outputs: one rounding of the value (half a step: 2^-8 of it in bf16, 2^-24 in float32), and in front of it what
    the sums leave. Prompts of bf16 round the state, or a token's update and the product of its key with the query, to
    f16 as operands: at most two roundings of 2^-11, relative to `sizes`, which is 2^-10, a quarter of 2^-8; the rest,
    float32 sums and operands of 22 bits, stays below a twentieth of 2^-8. In float32 operands have 22 bits (a product is
    off by 2^-21 at most), sums up to 256 values, and the errors of as many steps of the recurrence as a test has between
    two resets by the decay add up: 128 times 2^-24."""
    half = 2.0 ** -8 if act == "bf16" else 2.0 ** -24
    return half * np.abs(want) + (0.3 * half if act == "bf16" else 128 * half) * sizes + 1e-30


def state_bound(want, act):
    """States are float32 whatever the activations: 128 times 2^-24 of the largest value of a head's state, a bound
    on what its entries are summed from."""
    return 128 * 2.0 ** -24 * np.abs(want).max((-1, -2), keepdims=True) + 1e-30


def near(got, want, tol, what):
    assert np.isfinite(got).all(), f"{what}: {(~np.isfinite(got)).sum()} of {got.size} not finite"
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / tol):.2f} of the bound"
