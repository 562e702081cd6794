"""The paged attention cache of a hybrid stack and what reads it, as cases through the public
entry points, beside the same operators in elementary torch operations.

A case is a dict of plain values. ``listed()`` gives the fixed cases, ``draw(rng)`` one more of
the same ranges, ``prepare(case, seed)`` what a user's program holds before the call,
``run(state)`` one pass, ``exact(case, seed)`` the same outputs in float64. Where ``own`` is
false, ``run`` computes in float32 with torch and rounds once at the end.

Operators (``op``):
  append   the packed [q | k | v] projection: RMSNorm of every q and k head, rotation by the
           token's position, k and v written to their pages (in the activation type or in 8 bits
           with one float32 scale per token and head), q left for the attention
  read     cached tokens back into packed rows of the activation type
  prefill  causal attention of packed prompt chunks over the cached pages
  decode   attention of one new token of every sequence over the cached pages

Activations are N(0, 1), as they leave a norm; head layouts are one of two ranks of the
3584-wide hybrid stack (16 heads of 112) and generic grouped-query ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_EPS = 1e-5
_BASE = 10000.0
_SPARE = 3                 # pages of the pool that no sequence names
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(name, op, act, kv, heads, page, **kw):
    c = dict(op=op, act=act, kv=kv, hq=heads[0], hkv=heads[1], d=heads[2], page=page, window=0, mix=0)
    c.update(kw)
    if name:
        c["name"] = name
    return c


_HYBRID = (16, 16, 112)    # one of two ranks of 32 heads over 3584 columns
_GQA = (32, 8, 128)


def listed():
    return [
        # the smallest call: one user's next token through the norm, the rotation and the cache
        _case("append_b1_bf16", "append", "bf16", "act", _GQA, 64, q="1", ctx="2310", norm=True, rot=128, inter=False),
        # one chunk of the chunked serving schedule into an 8-bit cache: the end of one prompt, one
        # whole prompt and the start of a third
        _case("append_chunk2048_fp8", "append", "bf16", "fp8", _HYBRID, 64, q="317,1130,601", ctx="4096,0,0", norm=True,
              rot=112, inter=False),
        # prefixes of several sequences handed to another instance, from an 8-bit cache
        _case("read_fp8_24000", "read", "bf16", "fp8", _GQA, 64, q="9000,14001,999", ctx="0,0,0"),
        # one short prompt's cached tokens
        _case("read_bf16_391", "read", "bf16", "act", _HYBRID, 16, q="391", ctx="0"),
        # the attention of that chunk of the serving schedule, at both activation types
        _case("prefill_chunk2048_bf16", "prefill", "bf16", "act", _HYBRID, 64, q="317,1130,601", ctx="4096,0,0"),
        _case("prefill_chunk2048_f32", "prefill", "f32", "act", _HYBRID, 64, q="317,1130,601", ctx="4096,0,0"),
        # the largest: one long prompt
        _case("prefill_8192_bf16", "prefill", "bf16", "act", _GQA, 64, q="8192", ctx="0"),
        # a short follow-up question behind a long document, in an 8-bit cache: few rows, long cache
        _case("prefill_33_ctx40000_fp8", "prefill", "bf16", "fp8", _GQA, 64, q="33", ctx="40000"),
        # one user's next token after a short prompt in the paper's default precision
        _case("decode_b1_ctx391_f32", "decode", "f32", "act", _HYBRID, 16, q="1", ctx="390"),
        # one user's next token behind a very long context
        _case("decode_b1_ctx131072_bf16", "decode", "bf16", "act", _GQA, 64, q="1", ctx="131071"),
        # a serving batch of ragged lengths on an 8-bit cache
        _case("decode_b64_ragged_fp8", "decode", "bf16", "fp8", _GQA, 64, q="64x1", ctx="64:200-8192", mix=1),
        # decode-heavy serving of many short contexts on one of two ranks of the hybrid stack
        _case("decode_b256_ctx768_bf16", "decode", "bf16", "act", _HYBRID, 64, q="256x1", ctx="256:512-1024", mix=2),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    op = rng.choice(["append", "read", "prefill", "prefill", "decode", "decode"])
    heads = rng.choice([_HYBRID, _GQA, (8, 8, 64), (24, 4, 128), (12, 2, 64), (16, 2, 256), (8, 1, 96), (20, 4, 80), (32, 2, 128)])
    act = "f32" if rng.random() < 0.2 else "bf16"
    kv = "act" if act == "f32" else rng.choice(["act", "fp8", "act", "fp8", "int8" if op in ("prefill", "decode") else "fp8"])
    c = _case("", op, act, kv, heads, rng.choice([16, 32, 64, 128]), mix=rng.randrange(1 << 20))
    if op == "decode":
        n = log(1, 128)
        most = min(65536, (1 << 18) // n)
        lo = log(1, most)
        c.update(q="%dx1" % n, ctx="%d:%d-%d" % (n, lo, log(lo, most)))
    else:
        n = log(1, 12)
        total = {"append": log(1, 8192), "read": log(1, 16384), "prefill": log(n, 2500)}[op]
        cuts = sorted(rng.randrange(total + 1) for _ in range(n - 1))
        q = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        ctx = [log(1, 6000) - 1 if rng.random() < 0.6 else 0 for _ in q]
        c.update(q=",".join(map(str, q)), ctx=",".join(map(str, ctx if op != "read" else [0] * n)))
    if op == "append":
        c.update(norm=rng.random() < 0.7, rot=rng.choice([heads[2], heads[2] // 2 // 8 * 8, 0]), inter=rng.random() < 0.4)
    if op in ("prefill", "decode") and rng.random() < 0.25:
        c["window"] = log(1, 3000)
    return c


# ------------------------------------------------------------------- sizes of a case
def _lens(c):
    """(tokens of this call, tokens cached before it) of every sequence."""
    t = c["q"]
    q = [1] * int(t.split("x")[0]) if "x" in t else [int(v) for v in t.split(",")]
    if ":" in c["ctx"]:  # "n:lo-hi": n lengths spread over lo .. hi
        lo, hi = (int(v) for v in c["ctx"].split(":")[1].split("-"))
        r = random.Random(c["mix"])
        ctx = [r.randint(lo, hi) for _ in q]
    else:
        ctx = [int(v) for v in c["ctx"].split(",")]
    return q, ctx


def _pairs(m, n, window):
    """Visible (query, key) pairs of m queries behind n cached tokens."""
    full = m * n + m * (m + 1) // 2
    if not window:
        return full
    return sum(min(n + i + 1, window) for i in range(m))


def work(c):
    q, ctx = _lens(c)
    T, hq, hkv, d = sum(q), c["hq"], c["hkv"], c["d"]
    s = 2 if c["act"] == "bf16" else 4
    kvb = hkv * (2 * d * s if c["kv"] == "act" else 2 * d + 8)   # one cached token, k and v
    if c["op"] == "append":
        return {"bytes": T * ((2 * hq + 2 * hkv) * d * s + kvb), "flops": T * (hq + hkv) * d * 10}
    if c["op"] == "read":
        return {"bytes": T * (kvb + 2 * hkv * d * s), "flops": 0 if c["kv"] == "act" else 2 * T * hkv * d}
    w = c["window"]
    seen = sum((m + n if not w else min(m + n, m + w - 1)) for m, n in zip(q, ctx) if m)
    return {"bytes": 2 * T * hq * d * s + seen * kvb, "flops": 4 * d * hq * sum(_pairs(m, n, w) for m, n in zip(q, ctx))}


# ------------------------------------------------------------------- inputs
_CODE = {"fp8": (448.0, torch.float8_e4m3fn), "int8": (127.0, torch.int8)}


def _quantise(x, kv):
    """Codes and the scale per row of 8-bit caching: x * (Q / max|x|) rounded to even, max|x| / Q."""
    Q, t = _CODE[kv]
    amax = x.abs().amax(-1, keepdim=True)
    inv = torch.where(amax > 0, Q / amax, torch.zeros_like(amax))
    y = (x * inv).clamp(-Q, Q)
    return (y.round() if kv == "int8" else y).to(t), (amax / Q).squeeze(-1)


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    act = _TYPE[c["act"]]
    q, ctx = _lens(c)
    n, T, ps, hkv, d = len(q), sum(q), c["page"], c["hkv"], c["d"]
    kv_len = [a + b for a, b in zip(q, ctx)]
    per = [-(-v // ps) for v in kv_len]
    width, used = max(1, max(per)), sum(per)
    pages = used + _SPARE
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    lay = torch.zeros(n, width, dtype=torch.int64)
    at = 0
    for i, p in enumerate(per):
        lay[i, :p] = torch.arange(at, at + p)
        at += p
    s = {"c": c, "table": order[lay.cuda()].contiguous(), "pages": pages}
    s["kv_len"] = torch.tensor(kv_len, dtype=torch.int32, device="cuda")
    s["q_len"] = torch.tensor(q, dtype=torch.int32, device="cuda")
    s["cu"] = torch.tensor([sum(q[:i]) for i in range(n + 1)], dtype=torch.int32, device="cuda")

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def pool():
        shape = (pages, hkv, ps, d)
        if c["kv"] == "act":
            return (torch.zeros(shape, device="cuda") if c["op"] == "append" else rand(*shape)).to(act), None
        if c["op"] == "append":
            return torch.zeros(shape, dtype=torch.uint8, device="cuda").view(_CODE[c["kv"]][1]), torch.zeros(shape[:3], device="cuda")
        return _quantise(rand(*shape), c["kv"])

    s["k"], s["k_scale"] = pool()
    s["v"], s["v_scale"] = pool()
    if c["op"] == "append":
        s["qkv"] = rand(T, (c["hq"] + 2 * hkv) * d).to(act)
        s["q_w"], s["k_w"] = (1 + 0.1 * rand(d), 1 + 0.1 * rand(d)) if c["norm"] else (None, None)
        s["freq"] = _BASE ** (-torch.arange(c["rot"] // 2, dtype=torch.float64) * 2 / max(c["rot"], 1))
    elif c["op"] != "read":
        s["q"] = rand(T, c["hq"] * d).to(act)
    if own:
        _bind(s)
    return s


def _bind(s):
    """What a user's program keeps: descriptor, pool, metadata, output buffers, workspace, the marshalled call."""
    from paper_2602_21144_amd import binding as B
    c = s["c"]
    T, hq, hkv, d = int(s["cu"][-1]), c["hq"], c["hkv"], c["d"]
    ad = B.make_attn_desc(hq, hkv, d, c["page"], kv_format=c["kv"], act=c["act"], window=c["window"])
    pool = B.KvPool(ad, s["k"], s["v"], s["k_scale"], s["v_scale"])
    one = c["op"] == "decode" or set(_lens(c)[0]) == {1}
    meta = B.KvMeta(ad, None if one else s["cu"], s["kv_len"], s["table"], s["pages"])
    ws = B.workspace(B.attn_workspace_bytes(ad, T, meta.nseq))
    dev = dict(dtype=_TYPE[c["act"]], device="cuda")
    if c["op"] == "append":
        tr = B.QkTransform(ad, q_norm_w=s["q_w"], k_norm_w=s["k_w"], eps=_EPS, inv_freq=s["freq"], interleaved=c["inter"])
        s["out"] = {"q": torch.empty(T, hq * d, **dev), "k": s["k"], "v": s["v"]}
        s["call"] = B.bind("ssm_kv_append", ad, tr, s["qkv"], meta, pool, s["out"]["q"], ws)
    elif c["op"] == "read":
        s["out"] = {"k": torch.empty(T, hkv * d, **dev), "v": torch.empty(T, hkv * d, **dev)}
        s["call"] = B.bind("ssm_kv_read", ad, meta, pool, s["out"]["k"], s["out"]["v"], ws)
    else:
        s["out"] = {"o": torch.empty(T, hq * d, **dev)}
        s["call"] = B.bind("ssm_attn_" + c["op"], ad, s["q"], meta, pool, s["out"]["o"], ws)
    if c["op"] == "append" and c["kv"] != "act":
        s["out"].update(k_scale=s["k_scale"], v_scale=s["v_scale"])


def run(s):
    if own:
        s["call"]()
        return s["out"]
    return {"append": _append, "read": _read, "prefill": _attend, "decode": _attend}[s["c"]["op"]](s)


# ------------------------------------------------------------------- plain forms
def _rows(s):
    """(sequence, position) of every packed row."""
    T = int(s["c"]["q"].split("x")[0]) if "x" in s["c"]["q"] else sum(int(v) for v in s["c"]["q"].split(","))
    t = torch.arange(T, dtype=torch.int32, device="cuda")
    i = torch.searchsorted(s["cu"], t, right=True, out_int32=True) - 1
    return i, t - s["cu"][i] + (s["kv_len"] - s["q_len"])[i]


def _heads(x, w, pos, s, norm):
    """Norm and rotation of [T][heads][d] float32."""
    c = s["c"]
    if norm:
        x = x * (1 / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS)) * w
    rot = c["rot"]
    if rot:
        a = pos.double()[:, None] * s["freq"].cuda()
        cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]
        r = x[..., :rot]
        lo, hi = (r[..., 0::2], r[..., 1::2]) if c["inter"] else (r[..., :rot // 2], r[..., rot // 2:])
        lo, hi = lo * cos - hi * sin, hi * cos + lo * sin
        r = torch.stack([lo, hi], -1).flatten(-2) if c["inter"] else torch.cat([lo, hi], -1)
        x = torch.cat([r, x[..., rot:]], -1)
    return x


def _append(s):
    c = s["c"]
    T, hq, hkv, d, ps = s["qkv"].shape[0], c["hq"], c["hkv"], c["d"], c["page"]
    i, pos = _rows(s)
    q, k, v = s["qkv"].float().view(T, hq + 2 * hkv, d).split([hq, hkv, hkv], 1)
    q = _heads(q, s["q_w"], pos, s, c["norm"]).to(s["qkv"].dtype).view(T, hq * d)
    k = _heads(k, s["k_w"], pos, s, c["norm"])
    page, off = s["table"][i, pos // ps].long(), (pos % ps).long()
    out = {"q": q, "k": s["k"], "v": s["v"]}
    if c["kv"] == "act":
        s["k"][page, :, off] = k.to(s["k"].dtype)
        s["v"][page, :, off] = v.to(s["v"].dtype)
        return out
    kc, ks = _quantise(k, c["kv"])
    vc, vs = _quantise(v, c["kv"])
    s["k"].view(torch.uint8)[page, :, off] = kc.view(torch.uint8)
    s["v"].view(torch.uint8)[page, :, off] = vc.view(torch.uint8)
    s["k_scale"][page, :, off] = ks
    s["v_scale"][page, :, off] = vs
    return {**out, "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _cached(s, x, scale, page, off):
    y = x.view(torch.uint8)[page, :, off].view(x.dtype) if x.dtype == torch.float8_e4m3fn else x[page, :, off]
    return y.float() if scale is None else y.float() * scale[page, :, off].unsqueeze(-1)


def _read(s):
    i, pos = _rows(s)
    ps, act = s["c"]["page"], _TYPE[s["c"]["act"]]
    page, off = s["table"][i, pos // ps].long(), (pos % ps).long()
    return {"k": _cached(s, s["k"], s["k_scale"], page, off).to(act).flatten(1),
            "v": _cached(s, s["v"], s["v_scale"], page, off).to(act).flatten(1)}


def _dense(s, x, scale):
    """[sequences][kv heads][tokens][d] float32 of all pages in the table."""
    y = x.view(torch.uint8)[s["table"].long()].view(x.dtype) if x.dtype == torch.float8_e4m3fn else x[s["table"].long()]
    y = y.float() if scale is None else y.float() * scale[s["table"].long()].unsqueeze(-1)
    return y.transpose(1, 2).flatten(2, 3)


def _attend(s):
    c = s["c"]
    act, hq, hkv, d = _TYPE[c["act"]], c["hq"], c["hkv"], c["d"]
    m, rep = max(_lens(c)[0]), hq // hkv
    k, v = _dense(s, s["k"], s["k_scale"]), _dense(s, s["v"], s["v_scale"])
    n, L = k.shape[0], k.shape[2]
    t = torch.arange(m, device="cuda")
    row = (s["cu"][:-1, None] + t).clamp(max=s["q"].shape[0] - 1).long()                  # [n][m]
    q = s["q"].float().view(-1, hkv, rep, d)[row]                                         # [n][m][hkv][rep][d]
    q = q.permute(0, 2, 3, 1, 4).reshape(n, hkv, rep * m, d)
    z = (q @ k.transpose(2, 3)).mul_(d ** -0.5).view(n, hkv, rep, m, L)
    pos = (s["kv_len"] - s["q_len"])[:, None] + t
    j = torch.arange(L, device="cuda")
    see = j <= pos[..., None]
    if c["window"]:
        see &= j > pos[..., None] - c["window"]
    z.masked_fill_(~see[:, None, None], float("-inf"))
    z = z.sub_(z.amax(-1, keepdim=True)).exp_()
    z = z.div_(z.sum(-1, keepdim=True)).view(n, hkv, rep * m, L)
    o = (z @ v).view(n, hkv, rep, m, d).permute(0, 3, 1, 2, 4).reshape(n, m, hq * d)
    return {"o": o[t[None] < s["q_len"][:, None]].to(act)}


# ------------------------------------------------------------------- float64
def _e4m3(x):
    """x rounded to the nearest e4m3 value (ties to even), |x| <= 448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -30))).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def exact(c, seed):
    plain = dict(c)
    s = prepare(plain, seed)
    q, ctx = _lens(c)
    hq, hkv, d, ps = c["hq"], c["hkv"], c["d"], c["page"]
    table = s["table"].cpu().tolist()
    K, V = (x.float().double() if sc is None else x.float().double() * sc.double()[..., None]
            for x, sc in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])))

    def tokens(pool, i, n):
        """[hkv][n][d]: the first n cached tokens of sequence i."""
        return pool[table[i][:-(-n // ps)]].transpose(0, 1).reshape(hkv, -1, d)[:, :n]

    if c["op"] == "read":
        return {key: torch.cat([tokens(p, i, m).transpose(0, 1).reshape(m, hkv * d) for i, m in enumerate(q) if m])
                for key, p in (("k", K), ("v", V))}
    if c["op"] == "append":
        return _exact_append(c, s, q, ctx, table)
    x = s["q"].double().view(-1, hq, d)
    out, at = [], 0
    for i, (m, n) in enumerate(zip(q, ctx)):
        if not m:
            continue
        k, v = tokens(K, i, n + m), tokens(V, i, n + m)
        p = torch.arange(n, n + m, device="cuda")[:, None]
        j = torch.arange(n + m, device="cuda")[None]
        hidden = (j > p) | ((j <= p - c["window"]) if c["window"] else torch.zeros_like(j > p))
        o = torch.empty(m, hq, d, dtype=torch.float64, device="cuda")
        for h in range(hq):
            z = x[at:at + m, h] @ k[h // (hq // hkv)].T / math.sqrt(d)
            z[hidden] = -math.inf
            o[:, h] = torch.softmax(z, -1) @ v[h // (hq // hkv)]
        out.append(o.reshape(m, hq * d))
        at += m
    return {"o": torch.cat(out)}


def _exact_append(c, s, q, ctx, table):
    hq, hkv, d, ps, rot = c["hq"], c["hkv"], c["d"], c["page"], c["rot"]
    T = sum(q)
    x = s["qkv"].double().view(T, hq + 2 * hkv, d).clone()
    pos = torch.tensor([n + t for m, n in zip(q, ctx) for t in range(m)], dtype=torch.float64, device="cuda")
    if c["norm"]:
        for h, w in [(h, s["q_w"]) for h in range(hq)] + [(hq + h, s["k_w"]) for h in range(hkv)]:
            x[:, h] = x[:, h] / ((x[:, h] ** 2).sum(-1, keepdim=True) / d + _EPS).sqrt() * w.double()
    for f in range(rot // 2):
        a, b = (2 * f, 2 * f + 1) if c["inter"] else (f, f + rot // 2)
        ang = (pos * float(s["freq"][f]))[:, None]
        u, w = x[:, :hq + hkv, a].clone(), x[:, :hq + hkv, b].clone()
        x[:, :hq + hkv, a] = u * ang.cos() - w * ang.sin()
        x[:, :hq + hkv, b] = w * ang.cos() + u * ang.sin()
    page = torch.tensor([table[i][(n + t) // ps] for i, (m, n) in enumerate(zip(q, ctx)) for t in range(m)], device="cuda")
    off = torch.tensor([(n + t) % ps for m, n in zip(q, ctx) for t in range(m)], device="cuda")
    out = {"q": x[:, :hq].reshape(T, hq * d)}
    for key, y in (("k", x[:, hq:hq + hkv]), ("v", x[:, hq + hkv:])):
        full = torch.zeros(s[key].shape, dtype=torch.float64, device="cuda")
        if c["kv"] != "act":
            Q = _CODE[c["kv"]][0]
            amax = y.abs().amax(-1)
            scale = torch.zeros(full.shape[:3], dtype=torch.float64, device="cuda")
            scale[page, :, off] = amax / Q
            out[key + "_scale"] = scale
            y = y / amax.clamp(min=1e-300)[..., None] * Q
            y = _e4m3(y) if c["kv"] == "fp8" else torch.round(y)
        full[page, :, off] = y
        out[key] = full
    return out
