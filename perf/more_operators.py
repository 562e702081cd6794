"""The gated delta rule of a recurrent stack and the norms around its block, as cases through the public
entry points, beside the same operators in elementary torch operations.

A case is a dict of plain values. ``listed()`` gives the fixed cases, ``draw(rng)`` one more of
the same ranges, ``prepare(case, seed)`` what a user's program holds before the call,
``run(state)`` one pass, ``exact(case, seed)`` the same outputs in float64. Where ``own`` is
false, ``run`` computes in float32 with torch and rounds once at the end.

Operators (``op``):
  prefill  the gated delta rule over packed prompts: from the convolved [q | k | v] rows and the columns a
           (decay) and b (write strength) of the projection to the output rows, states of the sequences
           read where a prompt continues and written
  decode   one new token of every sequence, its state read and advanced in place, the norm of every head
           with its gate behind it where ``norm`` says so
  gnorm    the norm of every head of packed rows with a gate, columns of the same projection
  block    what lies between two blocks: the norm behind the first, its gate and scale, the residual add,
           the norm in front of the next

q, k and v are what a convolution with SiLU leaves of N(0, 1); a, b, z and gates N(0, 1); decays follow the Mamba-2
layer's initialisation (A from 1 to 16, step sizes from 1e-3 to 0.1).
"""
from __future__ import annotations

import math

import torch

own = False

_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS, _L2_EPS = 1e-5, 1e-6
_CHUNK = 64
_SPARE = 2                 # slots of the pool that no sequence names


def _delta(name, op, act, heads, q, init="", norm=False, l2=True, bmax=1.0):
    c = dict(op=op, act=act, hk=heads[0], hv=heads[1], dk=heads[2], dv=heads[3], q=q, init=init, norm=norm, l2=l2, bmax=bmax)
    return dict(c, name=name) if name else c


def _gnorm(name, act, rows, heads, dim, gate="silu", first=False, shared=True):
    c = dict(op="gnorm", act=act, rows=rows, heads=heads, dim=dim, gate=gate, first=first, shared=shared)
    return dict(c, name=name) if name else c


def _block(name, act, rows, dim, parts, gate="", fn="identity", post=True, scale=1.0):
    c = dict(op="block", act=act, rows=rows, dim=dim, parts=parts, gate=gate, fn=fn, post=post, scale=scale)
    return dict(c, name=name) if name else c


_RANK = (8, 16, 128, 128)     # one of two ranks of 16 query/key heads and 32 value heads of 128
_EQUAL = (12, 12, 64, 64)     # as many query/key heads as value heads, half the width


def listed():
    return [
        # the smallest call: one user's next token, the head norm with it
        _delta("decode_b1_bf16", "decode", "bf16", _RANK, "1x1", norm=True),
        # a serving batch's next tokens in the paper's default precision, wide values
        _delta("decode_b9_f32_96x192", "decode", "f32", (6, 6, 96, 192), "9x1", norm=True),
        # decode-heavy serving of many sequences
        _delta("decode_b256_bf16", "decode", "bf16", _RANK, "256x1", norm=True),
        # one short prompt in the paper's default precision
        _delta("prefill_391_f32", "prefill", "f32", _EQUAL, "391", "0"),
        # one chunk of the chunked serving schedule: the end of one prompt, one whole prompt and the start of a third
        _delta("prefill_chunk2048_bf16", "prefill", "bf16", _RANK, "317,1130,601", "1,0,0"),
        _delta("prefill_chunk2048_f32", "prefill", "f32", _RANK, "317,1130,601", "1,0,0"),
        # a batch of prompts of one length
        _delta("prefill_8x2048_bf16", "prefill", "bf16", _RANK, "2048," * 7 + "2048", "0," * 7 + "0"),
        # the largest: one long prompt of few heads and three more, the sequences of the long-prompt workload
        _delta("prefill_4x16384_bf16", "prefill", "bf16", _RANK, "16384,16384,16384,16384", "0,0,0,0"),
        # the head norm of one short prompt's rows, and of that chunk of the serving schedule
        _gnorm("gnorm_391_f32", "f32", 391, 12, 64),
        _gnorm("gnorm_16384_bf16", "bf16", 16384, 16, 128),
        # between two blocks: one decode step of a small batch, and two ranks' partials of a chunk with a gate per token
        _block("block_8x2560_bf16", "bf16", 8, 2560, 1),
        _block("block_2048x3584_gated_bf16", "bf16", 2048, 3584, 2, "token", "sigmoid", True, 0.5),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    op = rng.choice(["prefill", "prefill", "prefill", "decode", "decode", "gnorm", "block"])
    act = "f32" if rng.random() < 0.3 else "bf16"
    if op == "gnorm":
        return _gnorm("", act, log(1, 16384), rng.choice([1, 6, 12, 16, 20]), rng.choice([32, 48, 64, 112, 128, 192, 256]),
                      rng.choice(["silu", "sigmoid"]), rng.random() < 0.3, rng.random() < 0.5)
    if op == "block":
        return _block("", act, log(1, 4096), rng.choice([768, 1000, 2560, 3584, 4096, 5120, 7168]), rng.choice([0, 1, 1, 2, 4]),
                      rng.choice(["", "token", "channel"]), rng.choice(["identity", "sigmoid", "tanh"]), rng.random() < 0.7,
                      rng.choice([1.0, 0.25]))
    heads = rng.choice([_RANK, _EQUAL, (6, 6, 96, 192), (4, 4, 256, 512), (2, 8, 64, 128), (8, 8, 112, 112), (1, 3, 80, 48),
                        (16, 32, 128, 128), (4, 20, 128, 64)])
    l2, bmax = rng.random() < 0.85, rng.choice([1.0, 1.0, 2.0])
    if op == "decode":
        return _delta("", "decode", act, heads, "%dx1" % log(1, min(256, (1 << 26) // (heads[1] * heads[2] * heads[3]))), norm=rng.random() < 0.6, l2=l2, bmax=bmax)
    n = log(1, 12)
    total = log(n, 8192)
    cuts = sorted(rng.randrange(total + 1) for _ in range(n - 1))
    q = [b - a for a, b in zip([0] + cuts, cuts + [total])]
    return _delta("", "prefill", act, heads, ",".join(map(str, q)), ",".join(str(int(rng.random() < 0.4)) for _ in q), l2=l2, bmax=bmax)


def _lens(c):
    return [1] * int(c["q"].split("x")[0]) if "x" in c["q"] else [int(v) for v in c["q"].split(",")]


def work(c):
    s = 2 if c["act"] == "bf16" else 4
    if c["op"] == "gnorm":
        n = c["rows"] * c["heads"] * c["dim"]
        return {"bytes": 3 * n * s, "flops": 10 * n}
    if c["op"] == "block":
        n = c["rows"] * c["dim"]
        gate = {"": 0, "token": n * s, "channel": c["dim"] * s}[c["gate"]]
        return {"bytes": n * (4 + c["parts"] * s + 4 + s) + gate, "flops": n * (10 + c["parts"])}
    q = _lens(c)
    T, n, hk, hv, dk, dv = sum(q), len(q), c["hk"], c["hv"], c["dk"], c["dv"]
    reads = n if c["op"] == "decode" else c["init"].split(",").count("1")
    rows = T * (2 * hk * dk + 2 * hv * dv + 2 * hv + (hv * dv if c["norm"] else 0)) * s
    return {"bytes": rows + (reads + n) * hv * dk * dv * 4, "flops": 6 * T * hv * dk * dv}


# ------------------------------------------------------------------- inputs
def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    act = _TYPE[c["act"]]

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    s = {"c": c}
    if c["op"] == "gnorm":
        n = c["heads"] * c["dim"]
        s["x"] = (0.3 * rand(c["rows"], n)).to(act)
        s["proj"] = rand(c["rows"], n + 8 * c["heads"]).to(act)     # z and what lies behind it
        s["w"] = 1 + 0.1 * rand(c["dim"] if c["shared"] else n)
    elif c["op"] == "block":
        s["base"] = rand(c["rows"], c["dim"])
        s["parts"] = [rand(c["rows"], c["dim"]).to(act) for _ in range(c["parts"])]
        s["post_w"] = 1 + 0.1 * rand(c["dim"]) if c["post"] else None
        s["norm_w"] = 1 + 0.1 * rand(c["dim"])
        s["gate"] = rand(c["rows"] if c["gate"] == "token" else 1, c["dim"]).to(act) if c["gate"] else None
    else:
        q, hv = _lens(c), c["hv"]
        T, n, wide = sum(q), len(q), hv * c["dv"]
        s["qkv"] = torch.nn.functional.silu(rand(T, 2 * c["hk"] * c["dk"] + wide)).to(act)
        if not c["l2"]:                                             # normalised by the program itself
            qk = s["qkv"][:, :2 * c["hk"] * c["dk"]].float().view(T, 2 * c["hk"], c["dk"])
            qk = qk / torch.sqrt((qk * qk).sum(-1, keepdim=True) + _L2_EPS)
            s["qkv"][:, :2 * c["hk"] * c["dk"]] = qk.flatten(1).to(act)
        s["proj"] = rand(T, -(-(wide + 2 * hv) // 8) * 8).to(act)   # columns z | b | a
        u = torch.rand(2, hv, generator=g, device="cuda")
        s["A_log"] = torch.log(1 + 15 * u[0])
        dt = torch.exp(math.log(1e-3) + u[1] * (math.log(0.1) - math.log(1e-3)))
        s["dt_bias"] = dt + torch.log(-torch.expm1(-dt))
        s["pool"] = 0.3 * rand(n + _SPARE, hv, c["dv"], c["dk"])
        s["slot"] = torch.randperm(n + _SPARE, generator=g, device="cuda")[:n].to(torch.int32)
        s["cu"] = torch.tensor([sum(q[:i]) for i in range(n + 1)], dtype=torch.int32, device="cuda")
        s["init"] = torch.tensor([1] * n if c["op"] == "decode" else [int(v) for v in c["init"].split(",")],
                                 dtype=torch.int32, device="cuda")
        s["w"] = 1 + 0.1 * rand(c["dv"]) if c["norm"] else None
    if own:
        _bind(s)
    return s


def _columns(s):
    """z, b and a in the projection."""
    wide, hv = s["c"]["hv"] * s["c"]["dv"], s["c"]["hv"]
    return s["proj"][:, :wide], s["proj"][:, wide:wide + hv], s["proj"][:, wide + hv:wide + 2 * hv]


def _bind(s):
    """What a user's program keeps: descriptor, metadata, output buffers, workspace, the marshalled call."""
    from paper_2602_21144_amd import binding as B
    c = s["c"]
    act = _TYPE[c["act"]]
    if c["op"] == "gnorm":
        norm = B.GatedNorm(s["w"], s["proj"][:, :c["heads"] * c["dim"]], c["heads"], c["dim"], eps=_EPS, gate=c["gate"], gate_first=c["first"])
        s["out"] = {"y": torch.empty_like(s["x"])}
        s["call"] = B.bind("ssm_gated_rmsnorm", s["x"], norm, s["out"]["y"])
        return
    if c["op"] == "block":
        s["out"] = {"residual": torch.empty_like(s["base"]), "normed": torch.empty_like(s["base"], dtype=act)}
        s["call"] = B.bind("ssm_block_rmsnorm", s["base"], s["parts"], s["out"]["residual"], s["norm_w"], _EPS, s["out"]["normed"],
                           post_w=s["post_w"], gate=s["gate"], gate_fn=c["fn"], scale=c["scale"])
        return
    dd = B.make_delta_desc(c["hk"], c["hv"], c["dk"], c["dv"], act=c["act"], qk_norm=c["l2"], norm_eps=_L2_EPS, beta_max=c["bmax"])
    gates = B.DeltaGates(dd, s["A_log"], s["dt_bias"])
    z, b, a = _columns(s)
    T, n = s["qkv"].shape[0], s["slot"].shape[0]
    s["out"] = {"o": torch.empty(T, c["hv"] * c["dv"], dtype=act, device="cuda"), "pool": s["pool"]}
    ws = B.workspace(B.delta_workspace_bytes(dd, T, n))
    if c["op"] == "decode":
        norm = B.GatedNorm(s["w"], z, c["hv"], c["dv"], eps=_EPS) if c["norm"] else None
        s["call"] = B.bind("ssm_delta_decode", dd, gates, s["qkv"], a, b, s["slot"], s["pool"], s["out"]["o"], ws, norm=norm)
    else:
        meta = B.SeqMeta(s["cu"].cpu().numpy(), s["slot"].cpu().numpy(), s["init"].cpu().numpy(), s["pool"].shape[0])
        s["call"] = B.bind("ssm_delta_prefill", dd, gates, s["qkv"], a, b, meta, s["pool"], s["out"]["o"], ws)


def run(s):
    if own:
        s["call"]()
        return s["out"]
    return {"prefill": _prefill, "decode": _decode, "gnorm": _gnorm_plain, "block": _block_plain}[s["c"]["op"]](s)


# ------------------------------------------------------------------- plain forms
def _fn(x, name):
    if name == "identity":
        return x
    if name == "tanh":
        return torch.tanh(x)
    y = 1 / (1 + torch.exp(-x))
    return x * y if name == "silu" else y


def _head_norm(x, w, z, gate="silu", first=False):
    """[rows][heads][dim] float32; w [dim] or [heads][dim]."""
    f = _fn(z, gate)
    x = x * f if first else x
    y = x * (1 / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS)) * w
    return y if first else y * f


def _gnorm_plain(s):
    c = s["c"]
    shape = (c["rows"], c["heads"], c["dim"])
    z = s["proj"][:, :c["heads"] * c["dim"]].float().reshape(shape)
    w = s["w"] if c["shared"] else s["w"].view(shape[1:])
    return {"y": _head_norm(s["x"].float().view(shape), w, z, c["gate"], c["first"]).flatten(1).to(s["x"].dtype)}


def _block_plain(s):
    c = s["c"]
    y = torch.zeros_like(s["base"]) if not s["parts"] else torch.stack([p.float() for p in s["parts"]]).sum(0)
    if c["post"]:
        y = y * (1 / torch.sqrt((y * y).mean(-1, keepdim=True) + _EPS)) * s["post_w"]
    if c["gate"]:
        y = y * _fn(s["gate"].float(), c["fn"])
    r = s["base"] + c["scale"] * y
    return {"residual": r, "normed": (r * (1 / torch.sqrt((r * r).mean(-1, keepdim=True) + _EPS)) * s["norm_w"]).to(_TYPE[c["act"]])}


def _heads(s):
    """q, k [T][value heads][dk] (normalised, q scaled), v, log decay (float64) and write strength of every row."""
    c = s["c"]
    T, hk, hv, dk, dv = s["qkv"].shape[0], c["hk"], c["hv"], c["dk"], c["dv"]
    q, k, v = s["qkv"].float().split([hk * dk, hk * dk, hv * dv], 1)
    q, k, v = q.reshape(T, hk, dk), k.reshape(T, hk, dk), v.reshape(T, hv, dv)
    if c["l2"]:
        q, k = (x * (1 / torch.sqrt((x * x).sum(-1, keepdim=True) + _L2_EPS)) for x in (q, k))
    q, k = (x.repeat_interleave(hv // hk, 1) for x in (q * dk ** -0.5, k))
    _, b, a = _columns(s)
    x = a.double() + s["dt_bias"].double()
    g = -torch.exp(s["A_log"].double()) * (torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs())))
    return q, k, v, g, c["bmax"] / (1 + torch.exp(-b.float()))


def _decode(s):
    c = s["c"]
    q, k, v, g, beta = _heads(s)
    S = s["pool"][s["slot"].long()] * torch.exp(g).float()[..., None, None]       # [n][hv][dv][dk]
    u = beta[..., None] * (v - (S @ k[..., None]).squeeze(-1))
    S = S + u[..., None] * k[..., None, :]
    o = (S @ q[..., None]).squeeze(-1)
    s["pool"][s["slot"].long()] = S
    if c["norm"]:
        o = _head_norm(o, s["w"], _columns(s)[0].float().reshape(o.shape))
    return {"o": o.flatten(1).to(s["qkv"].dtype), "pool": s["pool"]}


def _prefill(s):
    """In chunks: per chunk U = T (beta V - beta e^G K S^T) with T = (I + tril(beta e^(Gi - Gj) K K^T))^-1."""
    c = s["c"]
    q, k, v, g, beta = _heads(s)
    lens, n = _lens(c), s["slot"].shape[0]
    N = max(1, -(-max(lens) // _CHUNK))
    t = torch.arange(N * _CHUNK, device="cuda")
    there = t < (s["cu"][1:] - s["cu"][:-1])[:, None]                             # [n][tokens]
    row = (s["cu"][:-1, None] + t).clamp(max=q.shape[0] - 1).long()

    def chunks(x):
        """[T][heads]([d]) -> [n][heads][chunks][64]([d]), zeros behind a sequence."""
        y = x[row] * there.view(there.shape + (1,) * (x.dim() - 1)).to(x.dtype)
        return y.view((n, N, _CHUNK) + x.shape[1:]).movedim(3, 1)

    q, k, v, G, beta = chunks(q), chunks(k), chunks(v), chunks(g).cumsum(-1), chunks(beta)
    low = torch.ones(_CHUNK, _CHUNK, dtype=torch.bool, device="cuda").tril()
    decay = torch.where(low, G[..., :, None] - G[..., None, :], -math.inf).exp().float()
    A = (beta[..., None] * decay * (k @ k.transpose(-1, -2))).tril(-1)
    T = torch.eye(_CHUNK, device="cuda").expand(A.shape).contiguous()
    for i in range(1, _CHUNK):                                                    # rows of the inverse, all chunks at once
        T[..., i, :i] -= (A[..., i, None, :i] @ T[..., :i, :i]).squeeze(-2)
    eG = G.exp().float()[..., None]
    W, U0 = T @ (beta[..., None] * eG * k), T @ (beta[..., None] * v)
    P = decay * (q @ k.transpose(-1, -2))
    q, k = q * eG, k * (G[..., -1:] - G).exp().float()[..., None]
    last = G[..., -1].exp().float()[..., None, None]
    S = (s["pool"][s["slot"].long()] * s["init"].view(-1, 1, 1, 1)).transpose(-1, -2).contiguous()   # [n][hv][dk][dv]
    o = torch.empty_like(v)
    for i in range(N):                                                            # the states follow each other
        U = U0[:, :, i] - W[:, :, i] @ S
        o[:, :, i] = q[:, :, i] @ S + P[:, :, i] @ U
        S = last[:, :, i] * S + k[:, :, i].transpose(-1, -2) @ U
    s["pool"][s["slot"].long()] = S.transpose(-1, -2).contiguous()
    o = o.movedim(1, 3).reshape(n, N * _CHUNK, -1)
    return {"o": o[there].to(s["qkv"].dtype), "pool": s["pool"]}


# ------------------------------------------------------------------- float64
def exact(c, seed):
    s = prepare(dict(c), seed)
    if c["op"] == "gnorm":
        x, z = s["x"].double(), s["proj"].double()[:, :c["heads"] * c["dim"]]
        gate = torch.sigmoid(z) * (z if c["gate"] == "silu" else 1)
        y = x * gate if c["first"] else x
        rms = y.reshape(c["rows"], c["heads"], -1).square().mean(2).add(_EPS).sqrt().repeat_interleave(c["dim"], 1)
        w = s["w"].double().repeat(c["heads"]) if c["shared"] else s["w"].double()
        return {"y": y / rms * w * (1 if c["first"] else gate)}
    if c["op"] == "block":
        y = torch.zeros(c["rows"], c["dim"], dtype=torch.float64, device="cuda")
        for p in s["parts"]:
            y += p.double()
        if c["post"]:
            y = y / y.square().mean(1, keepdim=True).add(_EPS).sqrt() * s["post_w"].double()
        if c["gate"]:
            z = s["gate"].double()
            y = y * {"identity": z, "sigmoid": torch.sigmoid(z), "tanh": torch.tanh(z)}[c["fn"]]
        r = s["base"].double() + c["scale"] * y
        return {"residual": r, "normed": r / r.square().mean(1, keepdim=True).add(_EPS).sqrt() * s["norm_w"].double()}
    return _exact_delta(c, s)


def _exact_delta(c, s):
    """Token by token, the sequences side by side."""
    q_len, hk, hv, dk, dv = _lens(c), c["hk"], c["hv"], c["dk"], c["dv"]
    T, n, rep = sum(q_len), len(q_len), hv // hk
    x = s["qkv"].double()
    q, k = x[:, :hk * dk].reshape(T, hk, dk), x[:, hk * dk:2 * hk * dk].reshape(T, hk, dk)
    v = x[:, 2 * hk * dk:].reshape(T, hv, dv)
    if c["l2"]:
        q, k = q / (q.norm(dim=2, keepdim=True) ** 2 + _L2_EPS).sqrt(), k / (k.norm(dim=2, keepdim=True) ** 2 + _L2_EPS).sqrt()
    z, b, a = (t.double() for t in _columns(s))
    alpha = torch.exp(-s["A_log"].double().exp() * torch.nn.functional.softplus(a + s["dt_bias"].double(), threshold=700.0))
    beta = c["bmax"] * torch.sigmoid(b)
    pool = s["pool"].double()
    slot = s["slot"].long()
    S = pool[slot] * s["init"].double().view(-1, 1, 1, 1)
    o = torch.zeros(T, hv, dv, dtype=torch.float64, device="cuda")
    start = [sum(q_len[:i]) for i in range(n)]
    for t in range(max(q_len)):
        on = [i for i in range(n) if t < q_len[i]]
        at = torch.tensor([start[i] + t for i in on], device="cuda") if t == 0 or len(on) != len(was) else at + 1
        who = slice(None) if len(on) == n else torch.tensor(on, device="cuda")
        was = on
        kt, qt = k[at].repeat_interleave(rep, 1)[:, :, None], q[at].repeat_interleave(rep, 1)[:, :, None]
        P = S[who] * alpha[at][..., None, None]
        P = P + (beta[at][..., None] * (v[at] - (P * kt).sum(-1)))[..., None] * kt
        o[at] = (P * qt).sum(-1) / math.sqrt(dk)
        S[who] = P
    pool[slot] = S
    if c["norm"]:
        o = o / (o.square().mean(2, keepdim=True) + _EPS).sqrt() * s["w"].double() * torch.nn.functional.silu(z.reshape(T, hv, dv))
    return {"o": o.reshape(T, hv * dv), "pool": pool}
