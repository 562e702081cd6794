"""Shared by the attention tests: a paged pool on the host, laid out page by page, with what no sequence
holds poisoned, and its copy on the GPU."""
import numpy as np

from oracle import attention as oa


class Pages:
    """Sequences of kv_len tokens spread over pages in a random order; `share` first pages of sequence 1 are
    sequence 0's."""

    def __init__(self, rng, kv_len, page, spare=2, extra=1, share=0):
        per = [-(-n // page) for n in kv_len]
        self.num = sum(per) + spare
        order = rng.permutation(self.num)
        self.table = np.zeros((len(kv_len), max(per + [1]) + extra), np.int32)
        at = 0
        for i, p in enumerate(per):
            self.table[i, :p] = order[at:at + p]
            at += p
        if share:
            self.table[1, :share] = self.table[0, :share]
        self.kv_len, self.page = list(kv_len), page

    def where(self, seq, pos):
        return self.table[seq, pos // self.page], pos % self.page


def poisoned_pool(torch, ad_args, pages, rng, act, fmt, fill=True):
    """(host k, v [num][hkv][page][D] float64 as the kernels see them, device k, v, k_scale, v_scale). What no
    sequence holds is NaN (codes 0x7f and NaN scales); with fill False everything is."""
    hkv, D, page = ad_args["hkv"], ad_args["d"], pages.page
    shape = (pages.num, hkv, page, D)
    held = np.zeros((pages.num, page), bool)
    if fill:
        for i, n in enumerate(pages.kv_len):
            for p in range(n):
                pg, off = pages.where(i, p)
                held[pg, off] = True
    out, dev, sc = [], [], []
    for _ in range(2):
        x = rng.standard_normal(shape).astype(np.float32)
        m = held[:, None, :]
        if fmt == "act":
            t = torch.from_numpy(x).to(torch.bfloat16 if act == "bf16" else torch.float32)
            t[torch.from_numpy(np.broadcast_to(~m, shape[:3]).copy())] = float("nan")
            dev.append(t.cuda())
            sc.append(None)
            out.append(t.to(torch.float64).numpy())
        else:
            q, s = oa.quantise(x.astype(np.float64), fmt)
            s = np.where(m, s, np.nan).astype(np.float32)
            q = np.where(m[..., None], q, 127.0 if fmt == "int8" else np.nan)
            tdt = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
            dev.append(torch.from_numpy(q.astype(np.float32)).to(tdt).cuda())
            sc.append(torch.from_numpy(np.ascontiguousarray(s)).cuda())
            out.append(q * s.astype(np.float64)[..., None])
    return out, dev, sc


def tokens(pool, pages, seq, n):
    """[n][hkv][D]: the first n cached tokens of a sequence (missing pages: NaN)."""
    rows = []
    for p in range(n):
        pg, off = pages.where(seq, p)
        rows.append(pool[pg, :, off] if 0 <= pg < pool.shape[0] else np.full((pool.shape[1], pool.shape[3]), np.nan))
    return np.stack(rows) if rows else np.zeros((0, pool.shape[1], pool.shape[3]))


def attn_tol(o, ab, big, n, D, act, fmt):
    """What the stated arithmetic can be off by, value by value. Scores: products summed in float32 (D
    roundings) of magnitude `big`, the scale and the exponent's own multiply (4 more): an absolute error in
    the exponent of 2 (D + 4) 2^-24 big, so that much relative error of p (twice: l has it too). exp2 and the
    sums over n tokens: (2 n + 16) 2^-24. bf16: p rounded (2^-8 each) and the result rounded (2^-8)."""
    u = 2.0 ** -24
    rel = 4 * (D + 4) * u * big + (2 * n + 16) * u
    if fmt != "act":
        rel += 4 * u
    if act == "bf16":
        rel += 2.0 ** -8
    out = np.abs(o) * (2.0 ** -8 if act == "bf16" else u)
    return ab * rel * 1.01 + out + 1e-30
