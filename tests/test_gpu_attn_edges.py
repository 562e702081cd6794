"""Calls at the edges of what the paged attention cache accepts: device metadata that the host check would have
refused, windows whose pages are given back, values that are not finite, and the forms that only larger calls take."""
import numpy as np
import pytest

from attn_cases import Pages, attn_tol, poisoned_pool, tokens
from oracle import attention as oa

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def test_overlapping_sequences_of_many_tiles():
    """Every second of 2^15 sequences names all rows of the call, 2^31 tiles in all: the plan has room for the first
    ones, which are whole, and the status names the others."""
    from paper_2602_21144_amd import binding as B
    T, n, hq, D, page = 1 << 17, 1 << 15, 128, 16, 4096
    ad = B.make_attn_desc(hq, 1, D, page, window=1)
    torch.manual_seed(60)
    k, v = (torch.randn(T // page, 1, page, D, device="cuda").bfloat16() for _ in range(2))
    pool = B.KvPool(ad, k, v)
    table = np.zeros((n, T // page), np.int32)
    table[0] = np.arange(T // page)
    meta = B.KvMeta(ad, [0] + [T] * n, [T] + [0] * (n - 1), table, T // page)
    meta.cu.copy_(torch.tensor([0, T] * (n // 2) + [0], dtype=torch.int32))
    meta.kv_len.fill_(T)
    meta.page_table.copy_(torch.from_numpy(np.broadcast_to(table[0], table.shape).copy()))
    q = torch.randn(T, hq * D, device="cuda").bfloat16()
    out = torch.full_like(q, float("nan"))
    ws = B.workspace(B.attn_workspace_bytes(ad, T, n))
    B.ssm_attn_prefill(ad, q, meta, pool, out, ws)
    assert B.take_status(ws) == B.SSM_STATUS_BAD_SEQLENS
    # a window of one token: every row is its own token's v
    assert torch.equal(out.view(T, hq, D), v.view(T, 1, D).expand(T, hq, D))


def _t(act):
    return torch.bfloat16 if act == "bf16" else torch.float32


def _f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def _near(got, want, tol, what):
    assert np.isfinite(got).all(), f"{what}: {(~np.isfinite(got)).sum()} of {got.size} not finite"
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / tol):.2f} of the bound"


def _attend(heads, page, q_lens, ctx, act, fmt, window=0, decode=False, seed=0, slid_out=False, rows=None, gone=None):
    """The attention of a call against the oracle at every row, or at about `rows` of each sequence. slid_out: what no row
    of a sequence sees any more holds NaN values and scales, and pages of such tokens alone are named out of range. gone
    {sequence: pages}: these are named out of range as well, though rows see them, and their tokens do not exist.
    Rows behind the last sequence keep what they hold. Returns what it called with."""
    from paper_2602_21144_amd import binding as B
    hq, hkv, D = heads
    rng = np.random.default_rng(seed)
    kv_len = [a + b for a, b in zip(q_lens, ctx)]
    pages = Pages(rng, kv_len, page)
    (K, V), dev, scales = poisoned_pool(torch, dict(hkv=hkv, d=D), pages, rng, act, fmt)
    ad = B.make_attn_desc(hq, hkv, D, page, kv_format=fmt, act=act, window=window)
    T = sum(q_lens)
    meta = B.KvMeta(ad, None if decode else np.concatenate([[0], np.cumsum(q_lens)]), kv_len, pages.table, pages.num)
    if slid_out:
        table = pages.table.copy()
        for i, (m, n) in enumerate(zip(q_lens, kv_len)):
            first = max(0, n - m - window + 1)
            at = [pages.where(i, p) for p in range(first)]
            if at:
                pg, off = (torch.tensor([int(x[j]) for x in at], device="cuda") for j in range(2))
                for t, s in zip(dev, scales):
                    if s is None:
                        t[pg, :, off] = float("nan")
                    else:
                        t.view(torch.uint8)[pg, :, off] = 0x7f
                        s[pg, :, off] = float("nan")
            for p in range(first // page):
                table[i, p] = (-1, pages.num, 2 ** 31 - 1)[p % 3]
        meta.page_table.copy_(torch.from_numpy(table))
    for i, ps in (gone or {}).items():
        meta.page_table[i, ps] = pages.num
    pool = B.KvPool(ad, *dev, *scales)
    q = torch.from_numpy(rng.standard_normal((T, hq * D)).astype(np.float32)).to(_t(act)).cuda()
    out = torch.full((T + 3, hq * D), float("nan"), dtype=_t(act), device="cuda")
    ws = B.workspace(B.attn_workspace_bytes(ad, T, len(q_lens)))
    (B.ssm_attn_decode if decode else B.ssm_attn_prefill)(ad, q, meta, pool, out, ws)
    assert B.take_status(ws) == (B.SSM_STATUS_BAD_PAGE if gone else 0)
    assert torch.isnan(out[T:]).all(), "written behind the rows"
    qh, got = _f64(q).reshape(T, hq, D), _f64(out[:T]).reshape(T, hq, D)
    assert np.isfinite(got).all(), f"{(~np.isfinite(got)).sum()} of {got.size} values are not finite"
    at = 0
    for i, (m, n) in enumerate(zip(q_lens, kv_len)):
        if m == 0:
            continue
        sel = np.arange(m) if rows is None or m <= rows else np.unique(np.r_[0, 1, m - 2, m - 1, rng.integers(0, m, rows)])
        ok = np.array([p // page not in gone.get(i, ()) for p in range(n)]) if gone else None
        o, ab, big = oa.attend(qh[at + sel], tokens(K, pages, i, n), tokens(V, pages, i, n), n - m + sel, ad.scale, window, ok)
        _near(got[at + sel], o, attn_tol(o, ab, big, n, D, act, fmt), f"sequence {i}")
        at += m
    return B, ad, pool, meta, q, out, ws


FORMATS = [("bf16", "act"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "act"), ("f32", "fp8"), ("f32", "int8")]


# ------------------------------------------------------------------- tokens that slid out of the window
@pytest.mark.parametrize("act,fmt", FORMATS)
@pytest.mark.parametrize("heads", [(4, 2, 64), (2, 1, 96), (3, 1, 128), (2, 1, 160), (4, 2, 256)])
def test_prefill_sees_nothing_in_front_of_the_window(act, fmt, heads):
    """NaN in values, codes and scales of tokens that no row sees, and pages of them given back: the window's first token
    is at every place of a step of 64 and of a block of 16, and in a later tile and piece."""
    _attend(heads, 16, [1, 1, 5, 40], [199, 333, 127, 1000], act, fmt, window=50, seed=61, slid_out=True)
    _attend(heads, 16, [1, 2, 3], [63, 130, 96], act, fmt, window=33, seed=62, slid_out=True)


@pytest.mark.parametrize("act,fmt", FORMATS)
@pytest.mark.parametrize("window", [1, 15, 16, 17, 31, 64, 100])
def test_prefill_windows_that_begin_anywhere(act, fmt, window):
    _attend((2, 1, 64), 32, [1, 1, 2, 7], [64 + 13, 128, 200, 97], act, fmt, window=window, seed=63, slid_out=True)


@pytest.mark.parametrize("act,fmt", FORMATS)
@pytest.mark.parametrize("window", [1, 16, 17, 33, 50, 100])
def test_decode_sees_nothing_in_front_of_the_window(act, fmt, window):
    _attend((4, 2, 64), 16, [1] * 5, [199, 333, 127, 1000, 20], act, fmt, window=window, decode=True, seed=64, slid_out=True)


@pytest.mark.parametrize("decode", [False, True])
def test_page_out_of_the_pool_inside_the_window_is_reported(decode):
    """The first page with a visible token, of which the window takes the last one."""
    B, ad, pool, meta, q, out, ws = _attend((4, 2, 64), 16, [1, 1], [199, 333], "bf16", "act", window=40, decode=decode, seed=65)
    f = B.ssm_attn_decode if decode else B.ssm_attn_prefill
    for first, want in ((334 - 40 - 1) // 16 - 1, 0), ((334 - 40) // 16, B.SSM_STATUS_BAD_PAGE):
        keep = meta.page_table[1, first].item()
        meta.page_table[1, first] = -1
        f(ad, q, meta, pool, out, ws)
        assert B.take_status(ws) == want
        meta.page_table[1, first] = keep


@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("f32", "fp8")])
def test_pages_that_slid_out_are_used_again(act, fmt):
    """A pool of seven pages of 16 serves a sequence of 160 tokens with a window of 40, token by token after its prompt, and
    beside it one that starts on the pages that it gave back."""
    from paper_2602_21144_amd import binding as B
    hq, hkv, D, page, W, num = 4, 2, 32, 16, 40, 7
    rng = np.random.default_rng(66)
    ad = B.make_attn_desc(hq, hkv, D, page, kv_format=fmt, act=act, window=W)
    pool = B.empty_kv_pool(ad, num)
    for t in pool.tensors():
        if t is not None:
            t.view(torch.uint8).fill_(0xff)
    width = (hq + 2 * hkv) * D
    x = []
    for n in (160, 20):   # values that every format holds exactly: e4m3 ones of a row whose largest is 448, by 2^-7
        y = oa.round_e4m3(np.clip(60 * rng.standard_normal((n, hq + 2 * hkv, D)), -448, 448))
        y[..., 0] = 448
        x.append(torch.from_numpy((y * 2.0 ** -7).reshape(n, width).astype(np.float32)).to(_t(act)).cuda())
    q, out = ([torch.empty(t.shape[0], hq * D, dtype=_t(act), device="cuda") for t in x] for _ in range(2))
    free, table = list(range(num)), np.full((2, 10), -1, np.int32)
    ws = B.workspace(B.attn_workspace_bytes(ad, 64, 2))

    def call(lens, rows):
        """`rows` new tokens of each sequence, which has lens[i] of them then."""
        seqs = [i for i in range(2) if rows[i]]
        for i in seqs:
            first = max(0, lens[i] - rows[i] - W + 1) // page
            for p in range(first):
                if table[i, p] >= 0:
                    free.append(int(table[i, p]))
                    table[i, p] = -1
            for p in range((lens[i] - rows[i]) // page, -(-lens[i] // page)):
                if table[i, p] < 0:
                    table[i, p] = free.pop(0)
        one = all(rows[i] == 1 for i in seqs)
        cu = None if one else np.concatenate([[0], np.cumsum([rows[i] for i in seqs])])
        meta = B.KvMeta(ad, cu, [lens[i] for i in seqs], table[seqs], num)
        rows_of = lambda t: torch.cat([t[i][lens[i] - rows[i]:lens[i]] for i in seqs])  # noqa: E731
        qq, oo = (torch.empty(sum(rows), hq * D, dtype=_t(act), device="cuda") for _ in range(2))
        B.ssm_kv_append(ad, None, rows_of(x), meta, pool, qq, ws)
        (B.ssm_attn_decode if one else B.ssm_attn_prefill)(ad, qq, meta, pool, oo, ws)
        at = 0
        for i in seqs:
            q[i][lens[i] - rows[i]:lens[i]], out[i][lens[i] - rows[i]:lens[i]] = qq[at:at + rows[i]], oo[at:at + rows[i]]
            at += rows[i]
    n = [0, 0]
    for rows in [(48, 0), (20, 0), (5, 0)] + [(1, 0)] * 27 + [(7, 3)] + [(1, 1)] * 17 + [(36, 0)]:
        n = [a + b for a, b in zip(n, rows)]
        call(n, rows)
    assert n == [160, 20] and B.take_status(ws) == 0
    for i, m in enumerate(n):
        _, k, v = oa.append(_f64(x[i]), hq, hkv, range(m), None, None, 0.0, np.zeros(0), False)
        if fmt != "act":
            (k, sk), (v, sv) = oa.quantise(k, fmt), oa.quantise(v, fmt)
            k, v = k * sk[..., None], v * sv[..., None]
        o, ab, big = oa.attend(_f64(q[i]).reshape(m, hq, D), k, v, range(m), ad.scale, W)
        got = _f64(out[i]).reshape(m, hq, D)
        _near(got, o, attn_tol(o, ab, big, m, D, act, fmt), f"sequence {i}")


# ------------------------------------------------------------------- operands of one buffer
@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("f32", "int8")])
@pytest.mark.parametrize("rows", [[1, 1, 1], [40, 1, 9]])
def test_operands_as_columns_of_one_buffer(act, fmt, rows):
    """Disjoint columns of a buffer are operands like any others: q and out beside [q | k | v], k beside v."""
    from paper_2602_21144_amd import binding as B
    hq, hkv, D, page = 4, 2, 48, 16
    rng = np.random.default_rng(67)
    kv = [m + n for m, n in zip(rows, (0, 30, 100))]
    pages = Pages(rng, kv, page)
    _, dev, scales = poisoned_pool(torch, dict(hkv=hkv, d=D), pages, rng, act, fmt)
    ad = B.make_attn_desc(hq, hkv, D, page, kv_format=fmt, act=act)
    one = max(rows) == 1
    meta = B.KvMeta(ad, None if one else np.concatenate([[0], np.cumsum(rows)]), kv, pages.table, pages.num)
    T, w = sum(rows), (hq + 2 * hkv) * D
    x = torch.randn(T, w, device="cuda").to(_t(act))
    ws = B.workspace(B.attn_workspace_bytes(ad, T, 3))
    got = []
    for shared in (False, True):
        pool = B.KvPool(ad, *(t.clone() for t in dev), *(None if t is None else t.clone() for t in scales))
        new = lambda n: torch.full((T, n), float("nan"), dtype=_t(act), device="cuda")  # noqa: E731
        if shared:
            a, b = new(w + 2 * hq * D), new(2 * hkv * D)
            qkv, q, out = a[:, hq * D:hq * D + w], a[:, :hq * D], a[:, hq * D + w:]
            k, v = b[:, hkv * D:], b[:, :hkv * D]
        else:
            qkv, q, out, k, v = (new(n * D) for n in (hq + 2 * hkv, hq, hq, hkv, hkv))
        qkv.copy_(x)
        B.ssm_kv_append(ad, None, qkv, meta, pool, q, ws)
        (B.ssm_attn_decode if one else B.ssm_attn_prefill)(ad, q, meta, pool, out, ws)
        B.ssm_kv_read(ad, meta, pool, k, v, ws)
        assert torch.equal(qkv, x)
        got.append((q, out, k, v))
    assert B.take_status(ws) == 0
    for a, b in zip(*got):
        assert torch.isfinite(a).all() and torch.equal(a, b)


# ------------------------------------------------------------------- codes
@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["fp8", "int8"])
@pytest.mark.parametrize("size", [2.0 ** -90, 1.0, 2.0 ** 100])
def test_codes_are_the_stated_float32_ones(act, fmt, size):
    """Code for code and scale for scale the float32 form of the definition, x * (Q / max) and max / Q with every step
    rounded to nearest: values of few bits lie on ties wherever Q / max is a power of two."""
    from paper_2602_21144_amd import binding as B
    T, hkv, D, page = 2048, 4, 112, 64
    ad = B.make_attn_desc(4, hkv, D, page, kv_format=fmt, act=act)
    pages = Pages(np.random.default_rng(68), [T], page)
    g = torch.Generator().manual_seed(68)
    x = torch.randn(T, 3 * hkv * D, generator=g).bfloat16().float() * size
    x.view(T, 3 * hkv, D)[:100, :, 3] = 7 * size          # Q / max is 64 / size with fp8
    x.view(T, 3 * hkv, D)[100:200, :, 5] = -127 * size     # and 1 / size with int8
    x = x.to(_t(act))
    pool, q = B.empty_kv_pool(ad, pages.num), torch.empty(T, hkv * D, dtype=_t(act), device="cuda")
    meta = B.KvMeta(ad, [0, T], [T], pages.table, pages.num)
    ws = B.workspace(B.attn_workspace_bytes(ad, T, 1))
    B.ssm_kv_append(ad, None, x.cuda(), meta, pool, q, ws)
    assert B.take_status(ws) == 0
    Q = np.float32(oa.CODE_MAX[fmt])
    pg, off = (np.array([pages.where(0, p)[i] for p in range(T)]) for i in range(2))
    for h0, t, s in ((hkv, pool.k, pool.k_scale), (2 * hkv, pool.v, pool.v_scale)):
        y = x.float().numpy().reshape(T, 3 * hkv, D)[:, h0:h0 + hkv]
        top = np.abs(y).max(-1)
        assert np.array_equal(s.cpu().numpy()[pg, :, off], top / Q)
        z = np.clip(y * (Q / top)[..., None], -Q, Q)
        got = t.view(torch.uint8).cpu().numpy()[pg, :, off]
        if fmt == "fp8":
            want = torch.from_numpy(z).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        else:
            want = np.rint(z).astype(np.int8).view(np.uint8)
        assert np.array_equal(got, want), f"{(got != want).sum()} of {got.size} codes"


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["act", "fp8", "int8"])
@pytest.mark.parametrize("heads", [(2, 2, 16), (4, 2, 112), (2, 1, 256)])
@pytest.mark.parametrize("transform", [False, True])
def test_values_that_are_no_numbers_stay_visible(act, fmt, heads, transform):
    """NaN and infinities in rows of k and v: an 8-bit cache holds such a row as NaN, the activation type holds the value;
    rows beside it are as without it, and single tokens and prompts that see it are NaN."""
    from paper_2602_21144_amd import binding as B
    hq, hkv, D = heads
    T, page, g = 24, 16, hq // hkv
    ad = B.make_attn_desc(hq, hkv, D, page, kv_format=fmt, act=act)
    pages = Pages(np.random.default_rng(69), [T], page)
    w = (hq + 2 * hkv) * D
    clean = torch.from_numpy(np.random.default_rng(69).standard_normal((T, w)).astype(np.float32)).to(_t(act)).cuda()
    x = clean.clone()
    v = x.view(T, hq + 2 * hkv, D)
    hit = {3: (hq, float("nan")), 7: (hq + hkv, float("nan")), 11: (hq + 2 * hkv - 1, float("inf")), 15: (hq, float("-inf"))}
    for i, (t, (h, value)) in enumerate(hit.items()):
        v[t, h, (0, D - 1, D // 2, 5)[i]] = value
    v[19, hq + hkv, :] = float("nan")
    tr = None
    if transform:
        tr = B.QkTransform(ad, torch.ones(D, device="cuda"), torch.ones(D, device="cuda"), 1e-5, 10000.0 ** (-np.arange(D // 2) * 2.0 / D))
    ws = B.workspace(B.attn_workspace_bytes(ad, T, 1))
    meta = B.KvMeta(ad, [0, T], [T], pages.table, pages.num)
    res = []
    for rows in (clean, x):
        pool = B.empty_kv_pool(ad, pages.num)
        q, k, vv, o = (torch.zeros(T, n * D, dtype=_t(act), device="cuda") for n in (hq, hkv, hkv, hq))
        B.ssm_kv_append(ad, tr, rows, meta, pool, q, ws)
        B.ssm_kv_read(ad, meta, pool, k, vv, ws)
        B.ssm_attn_prefill(ad, q, meta, pool, o, ws)
        steps = []
        for n in (3, 4, 7, 8, T):
            od = torch.zeros(1, hq * D, dtype=_t(act), device="cuda")
            B.ssm_attn_decode(ad, q[n - 1:n], B.KvMeta(ad, None, [n], pages.table, pages.num), pool, od, ws)
            steps.append(od)
        assert B.take_status(ws) == 0
        res.append((q, k.view(T, hkv, D), vv.view(T, hkv, D), o.view(T, hq, D), torch.cat(steps).view(5, hq, D)))
    (q0, k0, v0, o0, s0), (q1, k1, v1, o1, s1) = res
    assert torch.equal(q0, q1)
    for which, a, b in (("k", k0, k1), ("v", v0, v1)):
        base = hq if which == "k" else hq + hkv
        lost = {(t, h - base) for t, (h, _) in hit.items() if base <= h < base + hkv} | ({(19, 0)} if which == "v" else set())
        for t in range(T):
            for h in range(hkv):
                if (t, h) not in lost:
                    assert torch.equal(a[t, h], b[t, h]), f"{which} of token {t}, head {h}"
                elif fmt == "act":
                    assert not torch.isfinite(b[t, h]).all()
                else:
                    assert torch.isnan(b[t, h]).all(), f"{which} of token {t}, head {h}"
    # heads of kv head 0 see token 3's k from row 3 on
    assert torch.isnan(o1[3:, :g]).all() and torch.isnan(s1[1:, :g]).all()
    assert torch.equal(s1[0], s0[0])


# ------------------------------------------------------------------- forms of larger calls
# Tiles of 256 rows by eight waves: bf16, heads of 97 to 128 values, 65536 rows of query heads and more
BF16 = [("bf16", "act"), ("bf16", "fp8"), ("bf16", "int8")]


@pytest.mark.parametrize("act,fmt", BF16)
@pytest.mark.parametrize("window", [0, 100, 700])
@pytest.mark.parametrize("heads,q,ctx", [
    ((128, 1, 128), [512], [0]),                        # the first call of this form, one kv head
    ((128, 1, 128), [1, 300, 0, 211, 5], [0, 900, 40, 0, 2000]),
    ((64, 8, 112), [1024], [3000]),                     # cut into items and joined
    ((64, 8, 112), [700, 1, 400], [0, 2500, 1111]),
    ((16, 16, 112), [2049, 0, 2081], [0, 7, 64]),       # last tiles of 1 and of 33 rows
    ((24, 8, 128), [2731, 5], [1, 4000]),
])
def test_tiles_of_256_rows(act, fmt, window, heads, q, ctx):
    assert sum(q) * heads[0] >= 65536
    _attend(heads, 32, q, ctx, act, fmt, window=window, seed=70, slid_out=window > 0, rows=14)


@pytest.mark.parametrize("fmt", ["act", "fp8"])
@pytest.mark.parametrize("rows", [1023, 1024, 1025])
def test_both_sides_of_the_taller_tiles(fmt, rows):
    _attend((64, 8, 112), 64, [rows - 40, 40], [100, 1500], "bf16", fmt, seed=71, rows=12)


@pytest.mark.parametrize("fmt", ["act", "int8"])
@pytest.mark.parametrize("window", [0, 500])
def test_tiles_of_256_rows_without_some_pages(fmt, window):
    _attend((64, 8, 128), 16, [1100], [300], "bf16", fmt, window=window, seed=72, rows=16, gone={0: [3, 21, 22, 40, 86]})


@pytest.mark.parametrize("act,fmt", FORMATS)
@pytest.mark.parametrize("heads", [(4, 2, 96), (6, 2, 112), (16, 4, 128), (2, 1, 160), (4, 2, 224), (5, 1, 256)])
def test_few_rows_behind_a_long_cache(act, fmt, heads):
    """Tiles that are cut into many items, at every padded width: the buffers of a step's scales go round."""
    for q, ctx in (([1], [4000]), ([33], [3000]), ([5, 3, 1], [2500, 1000, 1700])):
        _attend(heads, 32, q, ctx, act, fmt, seed=73, rows=10)


@pytest.mark.parametrize("decode", [False, True])
def test_many_pages_a_table_row(decode):
    """65536 tokens of one kv head, in the smallest pages."""
    _attend((3, 1, 32), 16, [1] if decode else [3], [65536], "bf16", "fp8", decode=decode, seed=74)


# ------------------------------------------------------------------- many tokens appended
@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("bf16", "fp8"), ("f32", "act"), ("f32", "int8")])
@pytest.mark.parametrize("rows,pos0", [((127,), (0,)), ((128,), (5,)), ((129,), (16,)), ((100, 1, 0, 156), (0, 40, 3, 17)),
                                       ((255, 1), (0, 0)), ((390,), (10,)), ((1500,), (3,))])
def test_append_of_many_tokens_against_the_oracle(act, fmt, rows, pos0):
    """Around and past the groups of 128 tokens that are dealt out to the XCDs: every token in its own place."""
    from test_gpu_attn import _append_case
    _append_case(act, fmt, (3, 1, 64), 0, False, False, pos0, rows=rows, seed=75)
    _append_case(act, fmt, (4, 2, 112), 32, True, True, pos0, rows=rows, seed=76, page=64)


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_append_of_many_wide_heads(act):
    from test_gpu_attn import _append_case
    _append_case(act, "fp8", (2, 1, 256), 64, False, True, (0, 2), rows=(200, 190), seed=77, page=32)


@pytest.mark.parametrize("act,fmt", FORMATS)
@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_as_large_as_stated(act, fmt, decode, sign):
    """Scaled scores of up to 0.97e9 (and down to that below 0), 1.5e7 apart: every row is the v of its largest score,
    though a score's float32 product with the exponent's factor is up to 64 off."""
    from paper_2602_21144_amd import binding as B
    n, D, page, hq = 64, 96, 16, 2
    ad = B.make_attn_desc(hq, 1, D, page, kv_format=fmt, act=act, scale=1.8)
    pool = B.empty_kv_pool(ad, n // page)
    table = np.arange(n // page)[None]
    x = torch.zeros(n, hq + 2, D)
    x[:, :hq, 0] = 2.0 ** 13 * sign
    x[:, hq, 0] = 2.0 ** 10 * torch.arange(1, n + 1)
    x[:, hq + 1] = torch.from_numpy(np.random.default_rng(78).choice([0.5, 1.0, 1.5, -1.75], (n, D)).astype(np.float32))
    x[:, hq + 1, 0] = 1.75                                  # the row's largest: the others are fp8 codes then
    x = x.view(n, -1).to(_t(act)).cuda()
    q, out, k, v = (torch.empty(n, w * D, dtype=_t(act), device="cuda") for w in (hq, hq, 1, 1))
    ws = B.workspace(B.attn_workspace_bytes(ad, n, 1))
    meta = B.KvMeta(ad, [0, n], [n], table, n // page)
    B.ssm_kv_append(ad, None, x, meta, pool, q, ws)
    B.ssm_kv_read(ad, meta, pool, k, v, ws)
    rows = range(n)
    if decode:
        for t in rows:
            B.ssm_attn_decode(ad, q[t:t + 1], B.KvMeta(ad, None, [t + 1], table, n // page), pool, out[t:t + 1], ws)
    else:
        B.ssm_attn_prefill(ad, q, meta, pool, out, ws)
    assert B.take_status(ws) == 0
    scores = np.float64(1.8) * 2.0 ** 13 * _f64(k)[:, 0]
    assert scores.max() < 1e9 and np.diff(scores).min() > 1e6
    want = np.stack([_f64(v)[t if sign > 0 else 0] for t in rows])[:, None].repeat(hq, 1)
    # the winner's p rounded once (bf16: 2^-8) and the result (2^-8); float32: product, sum, quotient
    tol = np.abs(want) * (2.1 * 2.0 ** -8 if act == "bf16" else 8 * 2.0 ** -24)
    _near(_f64(out).reshape(n, hq, D), want, tol, "the largest score's v")
