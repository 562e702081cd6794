"""The paged attention cache on the GPU against the float64 oracle: appended and read-back values, prompt and
single-token attention over every activation type, cache format, head layout, page size and window, with
whatever no sequence holds set to NaN; strides, padded batches, bad metadata, graphs, streams, and the chain
of them as a hybrid stack's attention layer runs it."""
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


def _t(act):
    return torch.bfloat16 if act == "bf16" else torch.float32


def _f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def _near(got, want, tol, what):
    got = np.asarray(got, np.float64)
    assert np.isfinite(got).all(), f"{what}: not finite"
    bad = np.abs(got - want) > tol
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.max(np.abs(got - want) / tol):.2f} of the bound"


def _strided(rows, cols, act, pad):
    """[rows][cols] inside a wider buffer whose other columns and last rows are NaN."""
    buf = torch.full((rows + 1, cols + pad), float("nan"), dtype=_t(act), device="cuda")
    return buf, buf[:rows, :cols]


def _attend_case(heads, page, q_lens, ctx, act, fmt, window=0, seed=0, pad=8, share=0, decode=False, scale=None,
                 powers=(0, 0)):
    from paper_2602_21144_amd import binding as B
    hq, hkv, D = heads
    rng = np.random.default_rng(seed)
    kv_len = [a + b for a, b in zip(q_lens, ctx)]
    pages = Pages(rng, kv_len, page, share=share)
    (K, V), (kd, vd), (ks, vs) = poisoned_pool(torch, dict(hkv=hkv, d=D), pages, rng, act, fmt)
    for x, dev, e in ((K, kd, powers[0]), (V, vd, powers[1])):   # exact: powers of two
        x *= 2.0 ** e
        if e:
            dev.mul_(2.0 ** e)
    ad = B.make_attn_desc(hq, hkv, D, page, kv_format=fmt, act=act, window=window, scale=scale)
    pool = B.KvPool(ad, kd, vd, ks, vs)
    T = sum(q_lens)
    cu = None if decode else np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    meta = B.KvMeta(ad, cu, kv_len, pages.table, pages.num)
    qbuf, q = _strided(T, hq * D, act, pad)
    q.copy_(torch.from_numpy(rng.standard_normal((T, hq * D)).astype(np.float32) * 2.0 ** -powers[0]))
    obuf, out = _strided(T, hq * D, act, pad)
    ws = B.workspace(B.attn_workspace_bytes(ad, T, len(q_lens)))
    (B.ssm_attn_decode if decode else B.ssm_attn_prefill)(ad, q, meta, pool, out, ws)
    assert B.take_status(ws) == 0
    assert torch.isnan(obuf[T:]).all() and torch.isnan(obuf[:, hq * D:]).all(), "written outside the rows"
    qh = _f64(q).reshape(T, hq, D)
    got = _f64(out).reshape(T, hq, D)
    at = 0
    for i, (m, n) in enumerate(zip(q_lens, ctx)):
        if m == 0:
            continue
        o, ab, big = oa.attend(qh[at:at + m], tokens(K, pages, i, n + m), tokens(V, pages, i, n + m), range(n, n + m),
                               ad.scale, window)
        _near(got[at:at + m], o, attn_tol(o, ab, big, n + m, D, act, fmt), f"sequence {i}")
        at += m
    return B, ad, pool, meta, q, out, ws


FORMATS = [("bf16", "act"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "act"), ("f32", "fp8"), ("f32", "int8")]
HEADS = [(2, 2, 16), (4, 2, 48), (3, 1, 64), (4, 2, 80), (2, 1, 96), (6, 2, 112), (4, 1, 128), (2, 2, 144), (2, 1, 192),
         (4, 2, 224), (5, 1, 256)]


# ------------------------------------------------------------------- decode
@pytest.mark.parametrize("act,fmt", FORMATS)
@pytest.mark.parametrize("heads", HEADS)
def test_decode_head_layouts(act, fmt, heads):
    _attend_case(heads, 16, [1] * 5, [0, 30, 31, 127, 300], act, fmt, decode=True, seed=1)


@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("bf16", "fp8"), ("f32", "act")])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("window", [0, 1, 33, 200])
def test_decode_pages_and_windows(act, fmt, page, window):
    _attend_case((4, 2, 64), page, [1] * 7, [0, 15, 16, 31, 128, 255, 700], act, fmt, window=window, decode=True, seed=2)


@pytest.mark.parametrize("g", [1, 2, 8, 15, 16, 17, 33, 64])
def test_decode_shared_heads(g):
    _attend_case((g, 1, 64), 32, [1, 1], [70, 259], "bf16", "act", decode=True, seed=3)


@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("bf16", "int8"), ("f32", "act")])
def test_decode_long_cache_is_split_and_joined(act, fmt):
    _attend_case((2, 1, 64), 64, [1], [20000], act, fmt, decode=True, seed=4)
    _attend_case((2, 1, 64), 64, [1, 1, 1], [9000, 3, 5000], act, fmt, window=4097, decode=True, seed=5)


def test_decode_many_short_sequences():
    rng = np.random.default_rng(6)
    _attend_case((2, 2, 32), 16, [1] * 300, list(rng.integers(0, 200, 300)), "bf16", "act", decode=True, seed=6)


# ------------------------------------------------------------------- prefill
@pytest.mark.parametrize("act,fmt", FORMATS)
@pytest.mark.parametrize("heads", HEADS)
def test_prefill_head_layouts(act, fmt, heads):
    _attend_case(heads, 16, [1, 37, 0, 130], [0, 30, 5, 64], act, fmt, seed=7)


@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("bf16", "fp8"), ("f32", "act")])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("window", [0, 1, 50, 129])
def test_prefill_pages_and_windows(act, fmt, page, window):
    _attend_case((4, 2, 64), page, [65, 1, 200], [0, 333, 77], act, fmt, window=window, seed=8)


@pytest.mark.parametrize("q,ctx", [([1], [0]), ([2], [700]), ([31], [1000]), ([33], [3000]), ([64], [64]), ([129], [4000]),
                                   ([5, 3, 1], [2500, 0, 1700])])
@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("bf16", "fp8"), ("f32", "act")])
def test_prefill_few_rows_behind_a_cache(q, ctx, act, fmt):
    _attend_case((4, 2, 64), 32, q, ctx, act, fmt, seed=9)


def test_prefill_of_single_rows_without_cu_seqlens_equals_decode():
    B, ad, pool, meta, q, out, ws = _attend_case((4, 2, 128), 32, [1] * 6, [0, 5, 64, 300, 31, 90], "bf16", "act", decode=True,
                                                 seed=10)
    o2 = torch.empty_like(out)
    B.ssm_attn_prefill(ad, q, meta, pool, o2, ws)
    # the same sums in another order, then one rounding each
    assert (o2.float() - out.float()).abs().max() <= 2 ** -6 * out.float().abs().max()


def test_shared_prefix_pages():
    _attend_case((4, 2, 64), 16, [3, 40], [61, 70], "bf16", "fp8", share=2, seed=11)
    _attend_case((4, 2, 64), 16, [1, 1], [64, 70], "bf16", "act", share=2, decode=True, seed=11)


def test_scores_of_any_size_and_scale():
    _attend_case((2, 1, 64), 16, [1, 1], [50, 200], "f32", "act", decode=True, seed=12, scale=6.0)
    _attend_case((2, 1, 64), 16, [40], [20], "f32", "act", seed=12, scale=6.0)
    _attend_case((2, 1, 64), 16, [40], [20], "f32", "act", seed=12, scale=1e-4)


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_prefill_of_many_sequences(act):
    """More sequences than the plan keeps in shared memory, most of them short or empty."""
    rng = np.random.default_rng(17)
    q = [int(x) for x in rng.integers(0, 4, 1500)]
    _attend_case((2, 1, 16), 16, q, [int(x) for x in rng.integers(0, 40, 1500)], act, "act", seed=17)


@pytest.mark.parametrize("decode", [False, True])
def test_window_wider_than_any_cache(decode):
    q = [1, 1] if decode else [50, 3]
    for window in (2 ** 31 - 1, 2 ** 31 - 40):
        _attend_case((2, 1, 64), 16, q, [3000, 10], "bf16", "act", window=window, decode=decode, seed=18)


# ------------------------------------------------------------------- rows and pages that hold nothing
@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("f32", "fp8")])
def test_padded_decode_batch(act, fmt):
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(13)
    kv = [9, 0, 40, 0]
    pages = Pages(rng, kv, 16)
    _, (kd, vd), (ks, vs) = poisoned_pool(torch, dict(hkv=2, d=32), pages, rng, act, fmt)
    ad = B.make_attn_desc(4, 2, 32, 16, kv_format=fmt, act=act)
    pool = B.KvPool(ad, kd, vd, ks, vs)
    meta = B.KvMeta(ad, None, kv, pages.table, pages.num)
    ws = B.workspace(B.attn_workspace_bytes(ad, 4, 4))
    qkv = torch.randn(4, 8 * 32, device="cuda").to(_t(act))
    q, out = torch.empty(4, 128, dtype=_t(act), device="cuda"), torch.full((4, 128), float("nan"), dtype=_t(act), device="cuda")
    keep = [t.view(torch.uint8).clone() for t in (kd, vd)]
    B.ssm_kv_append(ad, None, qkv, meta, pool, q, ws)
    B.ssm_attn_decode(ad, q, meta, pool, out, ws)
    o2 = torch.full_like(out, float("nan"))
    B.ssm_attn_prefill(ad, q, meta, pool, o2, ws)
    kr, vr = (torch.full((4, 64), float("nan"), dtype=_t(act), device="cuda") for _ in range(2))
    B.ssm_kv_read(ad, meta, pool, kr, vr, ws)
    assert B.take_status(ws) == 0
    for r in (out, o2):
        assert (r[[1, 3]] == 0).all() and torch.isfinite(r).all() and (r[[0, 2]] != 0).any()
    assert torch.isnan(kr[[1, 3]]).all() and torch.isfinite(kr[[0, 2]]).all() and torch.isfinite(vr[[0, 2]]).all()
    assert torch.equal(q.view(torch.uint8), qkv[:, :128].contiguous().view(torch.uint8))   # no transform: q as it came
    for old, t in zip(keep, (kd, vd)):   # exactly the two tokens changed
        diff = (old != t.view(torch.uint8)).view(pages.num, 2, 16, -1).any(-1).any(1).nonzero().cpu().numpy().tolist()
        assert sorted(diff) == sorted([list(pages.where(0, 8)), list(pages.where(2, 39))])


@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("bf16", "fp8"), ("f32", "act")])
def test_pages_outside_the_pool_are_left_out(act, fmt):
    """A table entry out of range, as a program's mistake leaves it: nothing is read or written there, the
    other tokens are attended as if those did not exist, and the status says so."""
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(14)
    q_lens, ctx, page, hq, hkv, D = [30, 1], [60, 200], 16, 4, 2, 64
    kv = [a + b for a, b in zip(q_lens, ctx)]
    pages = Pages(rng, kv, page)
    (K, V), (kd, vd), (ks, vs) = poisoned_pool(torch, dict(hkv=hkv, d=D), pages, rng, act, fmt)
    ad = B.make_attn_desc(hq, hkv, D, page, kv_format=fmt, act=act)
    pool = B.KvPool(ad, kd, vd, ks, vs)
    gone = {0: [1, 5], 1: [0, 7, 12]}
    for decode in (False, True):
        rows = [1, 1] if decode else q_lens
        meta = B.KvMeta(ad, None if decode else [0, 30, 31], kv, pages.table, pages.num)
        bad = pages.table.copy()
        for i, ps in gone.items():
            for j, p in enumerate(ps):
                bad[i, p] = (-1, pages.num, 2 ** 31 - 1)[j]
        meta.page_table.copy_(torch.from_numpy(bad))
        T = sum(rows)
        q = torch.randn(T, hq * D, device="cuda").to(_t(act))
        out = torch.full((T, hq * D), float("nan"), dtype=_t(act), device="cuda")
        ws = B.workspace(B.attn_workspace_bytes(ad, T, 2))
        (B.ssm_attn_decode if decode else B.ssm_attn_prefill)(ad, q, meta, pool, out, ws)
        assert B.take_status(ws) == B.SSM_STATUS_BAD_PAGE
        at = 0
        for i, m in enumerate(rows):
            n = kv[i]
            ok = np.array([p // page not in gone[i] for p in range(n)])
            o, ab, big = oa.attend(_f64(q)[at:at + m].reshape(m, hq, D), tokens(K, pages, i, n), tokens(V, pages, i, n),
                                   range(n - m, n), ad.scale, 0, ok)
            _near(_f64(out)[at:at + m].reshape(m, hq, D), o, attn_tol(o, ab, big, n, D, act, fmt), f"sequence {i}")
            at += m
    # append and read leave those tokens out
    meta = B.KvMeta(ad, [0, 30, 31], kv, pages.table, pages.num)
    bad = pages.table.copy()
    bad[0, 5] = pages.num          # tokens 80 .. 89 of sequence 0: its last ten rows
    meta.page_table.copy_(torch.from_numpy(bad))
    ws = B.workspace(B.attn_workspace_bytes(ad, 31, 2))
    kr, vr = (torch.full((31, hkv * D), float("nan"), dtype=_t(act), device="cuda") for _ in range(2))
    B.ssm_kv_read(ad, meta, pool, kr, vr, ws)
    assert B.take_status(ws) == B.SSM_STATUS_BAD_PAGE
    assert torch.isnan(kr[20:30]).all() and torch.isfinite(kr[:20]).all() and torch.isfinite(kr[30]).all()
    before = [t.view(torch.uint8).clone() for t in (kd, vd)]
    qkv = torch.randn(31, (hq + 2 * hkv) * D, device="cuda").to(_t(act))
    B.ssm_kv_append(ad, None, qkv, meta, pool, torch.empty(31, hq * D, dtype=_t(act), device="cuda"), ws)
    assert B.take_status(ws) == B.SSM_STATUS_BAD_PAGE
    for old, t in zip(before, (kd, vd)):
        n = (old != t.view(torch.uint8)).view(pages.num, hkv, page, -1).any(-1).any(1).sum().item()
        assert n == 21


def test_lengths_that_do_not_fit_leave_the_sequence_out():
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(15)
    pages = Pages(rng, [20, 40, 10], 16)
    _, (kd, vd), _ = poisoned_pool(torch, dict(hkv=1, d=16), pages, rng, "bf16", "act")
    ad = B.make_attn_desc(2, 1, 16, 16)
    pool = B.KvPool(ad, kd, vd)
    q = torch.randn(30, 32, device="cuda").bfloat16()
    good = torch.full((30, 32), float("nan"), dtype=torch.bfloat16, device="cuda")
    meta = B.KvMeta(ad, [0, 10, 20, 30], [20, 40, 10], pages.table, pages.num)
    ws = B.workspace(B.attn_workspace_bytes(ad, 30, 3))
    B.ssm_attn_prefill(ad, q, meta, pool, good, ws)
    assert B.take_status(ws) == 0 and torch.isfinite(good).all()
    for cu, kv, lost in (([0, 10, 20, 30], [20, 9, 10], slice(10, 20)), ([0, 10, 20, 30], [20, -3, 10], slice(10, 20)),
                         ([0, 10, 20, 30], [20, 2 ** 30, 10], slice(10, 20)), ([0, 10, 20, 31], [20, 40, 11], slice(20, 30)),
                         ([0, 10, 5, 30], [20, 40, 25], None), ([0, 30, 0, 30], [30, 40, 30], None),
                         ([-4, 10, 20, 30], [20, 40, 10], slice(0, 10))):
        meta.cu.copy_(torch.tensor(cu, dtype=torch.int32))
        meta.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        out = torch.full_like(good, float("nan"))
        kr = torch.full((30, 16), float("nan"), dtype=torch.bfloat16, device="cuda")
        B.ssm_attn_prefill(ad, q, meta, pool, out, ws)
        B.ssm_kv_read(ad, meta, pool, kr, torch.empty_like(kr), ws)
        assert B.take_status(ws) & B.SSM_STATUS_BAD_SEQLENS
        if lost is None:
            continue
        assert torch.isnan(out[lost]).all() and torch.isnan(kr[lost]).all()
        rest = torch.ones(30, dtype=torch.bool)
        rest[lost] = False
        assert torch.equal(out[rest], good[rest])
    # a negative length in a decode batch: that row stays as it was
    meta = B.KvMeta(ad, None, [20, 40, 10], pages.table, pages.num)
    meta.kv_len.copy_(torch.tensor([20, -1, 10], dtype=torch.int32))
    out = torch.full((3, 32), float("nan"), dtype=torch.bfloat16, device="cuda")
    B.ssm_attn_decode(ad, q[:3].contiguous(), meta, pool, out, ws)
    assert B.take_status(ws) == B.SSM_STATUS_BAD_SEQLENS
    assert torch.isnan(out[1]).all() and torch.isfinite(out[[0, 2]]).all()


def test_rows_behind_the_last_sequence_stay():
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(16)
    pages = Pages(rng, [20, 7], 16)
    _, (kd, vd), _ = poisoned_pool(torch, dict(hkv=1, d=32), pages, rng, "bf16", "act")
    ad = B.make_attn_desc(2, 1, 32, 16)
    pool = B.KvPool(ad, kd, vd)
    meta = B.KvMeta(ad, [0, 20, 27], [20, 7], pages.table, pages.num)
    meta.cu.copy_(torch.tensor([0, 20, 25], dtype=torch.int32))
    meta.kv_len.copy_(torch.tensor([20, 5], dtype=torch.int32))
    ws = B.workspace(B.attn_workspace_bytes(ad, 27, 2))
    nan = lambda w: torch.full((27, w), float("nan"), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    q, out, kr, vr = nan(64), nan(64), nan(32), nan(32)
    B.ssm_kv_append(ad, None, torch.randn(27, 128, device="cuda").bfloat16(), meta, pool, q, ws)
    B.ssm_attn_prefill(ad, q, meta, pool, out, ws)
    B.ssm_kv_read(ad, meta, pool, kr, vr, ws)
    assert B.take_status(ws) == 0
    for t in (q, out, kr, vr):
        assert torch.isnan(t[25:]).all() and torch.isfinite(t[:25]).all()


@pytest.mark.parametrize("powers", [(40, -60), (-60, 100), (-100, 0)])
@pytest.mark.parametrize("decode", [False, True])
def test_float32_values_of_any_magnitude(powers, decode):
    """Scores of order one from factors far apart, small and large v: the parts of a value keep its 24 bits."""
    _attend_case((4, 2, 112), 16, [1, 1] if decode else [70, 33], [300, 20], "f32", "act", decode=decode, seed=15, powers=powers)


# ------------------------------------------------------------------- append and read
def _append_case(act, fmt, heads, rot, inter, norm, pos0, page=16, rows=(5, 1, 9), in_place=False, seed=20, scale_x=1.0):
    from paper_2602_21144_amd import binding as B
    hq, hkv, D = heads
    rng = np.random.default_rng(seed)
    kv = [r + p for r, p in zip(rows, pos0)]
    pages = Pages(rng, [min(k, 400) for k in kv], page) if max(kv) <= 400 else None
    if pages is None:   # far positions: a table whose early pages all name page 0
        per = [-(-k // page) for k in kv]
        table = np.zeros((len(kv), max(per)), np.int32)
        at = 1
        for i, (k, p) in enumerate(zip(kv, pos0)):
            for j in range(p // page, per[i]):
                table[i, j] = at
                at += 1
        num = at
        where = lambda i, p: (table[i, p // page], p % page)  # noqa: E731
    else:
        table, num, where = pages.table, pages.num, pages.where
    ad = B.make_attn_desc(hq, hkv, D, page, kv_format=fmt, act=act)
    pool = B.empty_kv_pool(ad, num)
    for t in (pool.k, pool.v):
        t.view(torch.uint8).fill_(0x5a)
    T = sum(rows)
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    meta = B.KvMeta(ad, cu, kv, table, num)
    W = (hq + 2 * hkv) * D
    buf, qkv = _strided(T, W, act, 16)
    x = rng.standard_normal((T, W)).astype(np.float32) * scale_x
    qkv.copy_(torch.from_numpy(x))
    x = _f64(qkv)
    qw, kw = ((1 + 0.2 * rng.standard_normal(D)).astype(np.float32) for _ in range(2)) if norm else (None, None)
    rad = 10000.0 ** (-np.arange(rot // 2) * 2.0 / max(rot, 1))
    tr = B.QkTransform(ad, None if qw is None else torch.from_numpy(qw).cuda(), None if kw is None else torch.from_numpy(kw).cuda(),
                       1e-5, rad, inter)
    q = qkv[:, :hq * D] if in_place else torch.empty(T, hq * D, dtype=_t(act), device="cuda")
    ws = B.workspace(B.attn_workspace_bytes(ad, T, len(rows)))
    B.ssm_kv_append(ad, tr, qkv, meta, pool, q, ws)
    kr, vr = (torch.empty(T, hkv * D + 8, dtype=_t(act), device="cuda")[:, :hkv * D] for _ in range(2))
    B.ssm_kv_read(ad, meta, pool, kr, vr, ws)
    assert B.take_status(ws) == 0
    pos = [p + r for n, p in zip(rows, pos0) for r in range(n)]
    seq = [i for i, n in enumerate(rows) for _ in range(n)]
    qo, ko, vo = oa.append(x, hq, hkv, pos, None if qw is None else qw.astype(np.float64),
                           None if kw is None else kw.astype(np.float64), 1e-5, rad, inter)
    # float32 steps: the norm's sum of D squares, root, divide and two multiplies ((D + 8) 2^-24 of the value);
    # the rotation's two products and their sum, with cosine and sine 4 2^-24 and the angle's 2^-31 off
    u = 2.0 ** -24
    half = 2.0 ** -8 if act == "bf16" else u
    rowmax = lambda y: np.abs(y).max(-1, keepdims=True)  # noqa: E731

    def tol(y, moved):
        return np.abs(y) * half + (rowmax(y) * ((D + 8 if norm else 0) + (16 if rot else 0)) * u if moved else 0) + 1e-37
    _near(_f64(q).reshape(T, hq, D), qo, tol(qo, True), "q")
    for name, ref, dev, scales, read, moved in (("k", ko, pool.k, pool.k_scale, kr, True), ("v", vo, pool.v, pool.v_scale, vr, False)):
        got = _f64(read).reshape(T, hkv, D)
        if fmt == "act":
            _near(got, ref, tol(ref, moved), name)
            stored = np.stack([_f64(dev)[where(s, p)[0], :, where(s, p)[1]] for s, p in zip(seq, pos)])
            assert np.array_equal(stored, got), f"{name}: what is read back is not what is stored"
            continue
        codes = dev.view(torch.uint8).cpu().numpy()
        cv = np.stack([oa.decode_codes(codes[where(s, p)[0], :, where(s, p)[1]], fmt) for s, p in zip(seq, pos)])
        sc = np.stack([scales.cpu().numpy()[where(s, p)[0], :, where(s, p)[1]] for s, p in zip(seq, pos)]).astype(np.float64)
        want_c, want_s = oa.quantise(ref, fmt)
        arith = ((D + 8 if norm else 0) + (16 if rot else 0) if moved else 0) * u
        _near(sc, want_s, want_s * (arith + 4 * u) * 1.5 + 1e-45, name + " scale")
        # half a step of the code in the row's scale, and the float32 arithmetic in front of it
        Q = oa.CODE_MAX[fmt]
        exact = np.where(want_s[..., None] > 0, ref / np.where(want_s > 0, want_s, 1)[..., None], 0.0)
        step = np.maximum(np.abs(exact) * 2.0 ** -4, 2.0 ** -10) if fmt == "fp8" else 0.5
        _near(cv, exact, step * (1 + 1e-6) + Q * (arith * 2 + 6 * u), name + " codes")
        assert np.abs(cv).max() <= Q
        _near(got, cv * sc[..., None], np.abs(cv * sc[..., None]) * (half + u) + 1e-45, name + " read back")
        if not moved:   # nothing but the quantisation: the codes are the oracle's where no tie is near
            # (a value between 2^e and 2^(e+1) is at most 2^(e-4) from its e4m3 code: 336, halfway between 320
            # and 352, lies 16 from either, not the 21 of the relative bound 336 2^-4)
            with np.errstate(divide="ignore"):
                e = np.maximum(np.floor(np.log2(np.abs(exact))), -6)
            tie = 2.0 ** (e - 4) if fmt == "fp8" else 0.5
            clear = np.abs(exact - want_c) < 0.9 * tie
            assert np.array_equal(cv[clear], want_c[clear])
    # everything else in the pool is as it was
    held = np.zeros((num, page), bool)
    for s, p in zip(seq, pos):
        held[where(s, p)] = True
    for dev in (pool.k, pool.v):
        raw = dev.view(torch.uint8).cpu().numpy().reshape(num, hkv, page, -1)
        assert (raw.transpose(0, 2, 1, 3)[~held] == 0x5a).all()
    assert torch.isnan(buf[:, W:]).all() and torch.isnan(buf[T:]).all()
    if not in_place:
        assert np.array_equal(_f64(qkv), x), "the input changed"


@pytest.mark.parametrize("act,fmt", FORMATS)
@pytest.mark.parametrize("heads", HEADS)
def test_append_and_read_back(act, fmt, heads):
    D = heads[2]
    _append_case(act, fmt, heads, D, False, True, (0, 100, 3))


@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("f32", "act"), ("bf16", "fp8"), ("f32", "int8")])
@pytest.mark.parametrize("rot", [0, 8, 32, 64, 128])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_append_norms_and_rotations(act, fmt, rot, inter, norm):
    _append_case(act, fmt, (3, 1, 128), rot, inter, norm, (0, 17, 250), in_place=norm)


@pytest.mark.parametrize("inter", [False, True])
def test_rotation_at_far_positions(inter):
    _append_case("f32", "act", (2, 1, 64), 64, inter, False, (0, 131071, 1 << 20), page=256)


@pytest.mark.parametrize("scale_x", [0.0, 1e-36, 1e-20, 1e20])
@pytest.mark.parametrize("fmt", ["act", "fp8", "int8"])
def test_append_rows_of_any_magnitude(fmt, scale_x):
    _append_case("f32", fmt, (2, 2, 32), 0, False, False, (0, 1, 2), scale_x=scale_x)


@pytest.mark.parametrize("rows", [(1500,), (600, 1, 0, 700)])
def test_append_many_tokens(rows):
    """The form that takes a token's heads in one workgroup."""
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(30)
    pages = Pages(rng, list(rows), 64)
    ad = B.make_attn_desc(6, 2, 64, 64, kv_format="fp8")
    T = sum(rows)
    qkv = torch.randn(T, 10 * 64, device="cuda").bfloat16()
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    tr = B.QkTransform(ad, torch.ones(64, device="cuda"), torch.ones(64, device="cuda"), 1e-5, 10000.0 ** (-np.arange(32) / 32.0))
    ws = B.workspace(B.attn_workspace_bytes(ad, T, len(rows)))
    got = []
    for whole in (True, False):
        pool = B.empty_kv_pool(ad, pages.num)
        q = torch.empty(T, 6 * 64, dtype=torch.bfloat16, device="cuda")
        if whole:
            B.ssm_kv_append(ad, tr, qkv, B.KvMeta(ad, cu, list(rows), pages.table, pages.num), pool, q, ws)
        else:   # in chunks of up to 100 rows of one sequence: the form that spreads the heads
            for i, n in enumerate(rows):
                for a in range(0, n, 100):
                    b = min(n, a + 100)
                    m = B.KvMeta(ad, [0, b - a], [b], pages.table[i:i + 1], pages.num)
                    B.ssm_kv_append(ad, tr, qkv[cu[i] + a:cu[i] + b], m, pool, q[cu[i] + a:cu[i] + b], ws)
        k, v = torch.empty(T, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(T, 128, dtype=torch.bfloat16, device="cuda")
        B.ssm_kv_read(ad, B.KvMeta(ad, cu, list(rows), pages.table, pages.num), pool, k, v, ws)
        got.append((q, k, v))
    assert B.take_status(ws) == 0
    for a, b in zip(*got):
        assert torch.equal(a, b)


# ------------------------------------------------------------------- order of sums, graphs, streams
@pytest.mark.parametrize("decode", [False, True])
def test_same_call_same_bits(decode):
    B, ad, pool, meta, q, out, ws = _attend_case((4, 2, 64), 32, [1] * 3 if decode else [33, 1, 70], [3000, 40, 900], "bf16", "fp8",
                                                 decode=decode, seed=40)
    first = out.clone()
    f = B.ssm_attn_decode if decode else B.ssm_attn_prefill
    for _ in range(5):
        out.fill_(float("nan"))
        f(ad, q, meta, pool, out, ws)
        assert torch.equal(out, first)


def test_graph_of_decode_steps_follows_kv_len():
    """A captured append + decode + advance, replayed with eager work between: every replay equals the eager
    step of the same token."""
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(41)
    n, hq, hkv, D, page, steps = 3, 4, 2, 64, 16, 6
    start = [1, 30, 127]
    pages = Pages(rng, [s + steps for s in start], page)
    ad = B.make_attn_desc(hq, hkv, D, page)
    tr = B.QkTransform(ad, torch.ones(D, device="cuda"), None, 1e-5, 10000.0 ** (-np.arange(16) / 16.0))
    xs = torch.randn(steps, n, (hq + 2 * hkv) * D, device="cuda").bfloat16()
    base = torch.randn(pages.num, hkv, page, D, device="cuda").bfloat16()
    outs = []
    for graph in (False, True):
        pool = B.KvPool(ad, base.clone(), base.clone())
        meta = B.KvMeta(ad, None, start, pages.table, pages.num)
        ws = B.workspace(B.attn_workspace_bytes(ad, n, n))
        x, q = torch.empty_like(xs[0]), torch.empty(n, hq * D, dtype=torch.bfloat16, device="cuda")
        out = torch.empty_like(q)

        def step():
            meta.kv_len += 1
            B.ssm_kv_append(ad, tr, x, meta, pool, q, ws)
            B.ssm_attn_decode(ad, q, meta, pool, out, ws)
        got = []
        if graph:
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g = torch.cuda.CUDAGraph()
                x.copy_(xs[0])
                s.synchronize()
                with torch.cuda.graph(g, stream=s):
                    step()
            torch.cuda.current_stream().wait_stream(s)
        for t in range(steps):
            x.copy_(xs[t])
            g.replay() if graph else step()
            torch.cuda.synchronize()
            got.append(out.clone())
            _ = (out.float() * 2).sum().item()   # eager work between the replays
        assert B.take_status(ws) == 0
        outs.append((got, pool.k, pool.v))
    for a, b in zip(outs[0][0], outs[1][0]):
        assert torch.equal(a, b)
    assert torch.equal(outs[0][1], outs[1][1]) and torch.equal(outs[0][2], outs[1][2])


@pytest.mark.parametrize("act,fmt", [("bf16", "fp8"), ("f32", "act")])
def test_graphs_of_chunks_share_a_workspace(act, fmt):
    """Two captured chunks (append, attention, read-back), one of a single sequence and one of three, and a
    captured decode step, in one workspace: replayed in turn on other inputs, each equals its eager calls."""
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(43)
    hq, hkv, D, page = 6, 2, 112, 16
    ad = B.make_attn_desc(hq, hkv, D, page, kv_format=fmt, act=act)
    tr = B.QkTransform(ad, None, torch.ones(D, device="cuda"), 1e-5, 10000.0 ** (-np.arange(56) / 56.0))
    calls = [([150], [1000]), ([3, 40, 1], [0, 17, 700]), (None, [30, 260])]
    ws = B.workspace(max(B.attn_workspace_bytes(ad, 200, 4), 1))
    jobs = []
    for rows, ctx in calls:
        m = rows or [1] * len(ctx)
        kv = [a + b for a, b in zip(m, ctx)]
        pages = Pages(rng, kv, page)
        _, (kd, vd), (ks, vs) = poisoned_pool(torch, dict(hkv=hkv, d=D), pages, rng, act, fmt)
        pool = B.KvPool(ad, kd, vd, ks, vs)
        meta = B.KvMeta(ad, None if rows is None else np.concatenate([[0], np.cumsum(m)]), kv, pages.table, pages.num)
        T = sum(m)
        x = torch.randn(T, (hq + 2 * hkv) * D, device="cuda").to(_t(act))
        q, out, kr, vr = (torch.empty(T, n * D, dtype=_t(act), device="cuda") for n in (hq, hq, hkv, hkv))

        def run(meta=meta, pool=pool, x=x, q=q, out=out, kr=kr, vr=vr, rows=rows):
            B.ssm_kv_append(ad, tr, x, meta, pool, q, ws)
            (B.ssm_attn_decode if rows is None else B.ssm_attn_prefill)(ad, q, meta, pool, out, ws)
            B.ssm_kv_read(ad, meta, pool, kr, vr, ws)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            run()
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                run()
        torch.cuda.current_stream().wait_stream(s)
        jobs.append((run, g, x, (out, kr, vr)))
    for t in range(3):
        for run, g, x, outs in jobs:
            x.normal_()
            run()
            torch.cuda.synchronize()
            want = [o.clone() for o in outs]
            for o in outs:
                o.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            for a, b in zip(want, outs):
                assert torch.equal(a, b)
    assert B.take_status(ws) == 0


def test_calls_on_two_streams_with_their_own_workspaces():
    B, ad, pool, meta, q, out, ws = _attend_case((4, 2, 64), 32, [40, 300], [900, 100], "bf16", "act", seed=42)
    want = out.clone()
    s = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(out) for _ in s]
    wss = [B.workspace(ws.numel()) for _ in s]
    torch.cuda.synchronize()
    for _ in range(4):
        for st, o, w in zip(s, outs, wss):
            B.ssm_attn_prefill(ad, q, meta, pool, o, w, stream=st)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, want)


def test_offsets_past_32_bits():
    """A pool whose last pages lie beyond 4 GiB (values and bytes), named by the table."""
    from paper_2602_21144_amd import binding as B
    hq, hkv, D, page = 2, 1, 256, 4096
    num = (5 << 30) // (page * D * 2)      # 5 GiB of k, 5 GiB of v
    ad = B.make_attn_desc(hq, hkv, D, page)
    k, v = (torch.empty(num, hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pool = B.KvPool(ad, k, v)
    table = np.array([[num - 1], [num - 2]], np.int32)
    rows = [70, 33]
    meta = B.KvMeta(ad, [0, 70, 103], rows, table, num)
    ws = B.workspace(B.attn_workspace_bytes(ad, 103, 2))
    qkv = torch.randn(103, 4 * D, device="cuda").bfloat16()
    q, out = (torch.empty(103, hq * D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.ssm_kv_append(ad, None, qkv, meta, pool, q, ws)
    B.ssm_attn_prefill(ad, q, meta, pool, out, ws)
    kr, vr = (torch.empty(103, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.ssm_kv_read(ad, meta, pool, kr, vr, ws)
    one = B.KvMeta(ad, None, rows, table, num)
    od = torch.empty(2, hq * D, dtype=torch.bfloat16, device="cuda")
    last = torch.tensor([69, 102], device="cuda")
    B.ssm_attn_decode(ad, q[last].contiguous(), one, pool, od, ws)
    assert B.take_status(ws) == 0
    assert torch.equal(kr, qkv[:, 2 * D:3 * D]) and torch.equal(vr, qkv[:, 3 * D:])
    K, V, Q = _f64(kr).reshape(103, 1, D), _f64(vr).reshape(103, 1, D), _f64(q).reshape(103, hq, D)
    for a, n in ((0, 70), (70, 33)):
        o, ab, big = oa.attend(Q[a:a + n], K[a:a + n], V[a:a + n], range(n), ad.scale)
        _near(_f64(out)[a:a + n].reshape(n, hq, D), o, attn_tol(o, ab, big, n, D, "bf16", "act"), "prefill")
        _near(_f64(od)[int(a > 0)].reshape(hq, D), o[-1], attn_tol(o[-1], ab[-1], big, n, D, "bf16", "act"), "decode")


# ------------------------------------------------------------------- the chain
@pytest.mark.parametrize("act,fmt", [("bf16", "act"), ("bf16", "fp8"), ("f32", "act")])
def test_attention_layer_in_chunks_equals_the_whole(act, fmt):
    """A hybrid stack's attention layer as it is served: norm, [q | k | v] projection, append, attention and
    output projection of two prompts in chunks, then single tokens; against one float64 pass over each whole
    sequence that quantises the cache as the kernels do."""
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(50)
    dm, hq, hkv, D, page = 128, 4, 2, 32, 16
    a = _t(act)
    W = (hq + 2 * hkv) * D
    wqkv = torch.from_numpy((rng.standard_normal((W, dm)) / np.sqrt(dm)).astype(np.float32)).to(a).cuda()
    wout = torch.from_numpy((rng.standard_normal((dm, hq * D)) / np.sqrt(hq * D)).astype(np.float32)).to(a).cuda()
    qw, kw = (torch.from_numpy((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)).cuda() for _ in range(2))
    nw = torch.ones(dm, device="cuda")
    rad = 10000.0 ** (-np.arange(D // 2) * 2.0 / D)
    lens = [45, 70]
    x = [torch.from_numpy(rng.standard_normal((n, dm)).astype(np.float32)).to(a).cuda() for n in lens]
    pages = Pages(rng, lens, page)
    ad = B.make_attn_desc(hq, hkv, D, page, kv_format=fmt, act=act)
    tr = B.QkTransform(ad, qw, kw, 1e-5, rad)
    pool = B.empty_kv_pool(ad, pages.num)
    ws = B.workspace(B.attn_workspace_bytes(ad, 128, 2))
    got = [torch.empty(n, dm, dtype=a, device="cuda") for n in lens]
    mid = []   # (normed rows, qkv) per call, for the float64 pass

    def call(parts, decode):   # parts: (sequence, first, last)
        rows = torch.cat([x[i][f:e] for i, f, e in parts])
        T = rows.shape[0]
        res, h = torch.empty(T, dm, device="cuda"), torch.empty(T, dm, dtype=a, device="cuda")
        B.ssm_residual_rmsnorm(rows, [], res, nw, 1e-5, h)
        qkv, q, o, y = (torch.empty(T, w, dtype=a, device="cuda") for w in (W, hq * D, hq * D, dm))
        B.ssm_gemm_nt(h, wqkv, qkv)
        cu = None if decode else np.concatenate([[0], np.cumsum([e - f for _, f, e in parts])])
        meta = B.KvMeta(ad, cu, [e for _, _, e in parts], pages.table[[i for i, _, _ in parts]], pages.num)
        B.ssm_kv_append(ad, tr, qkv, meta, pool, q, ws)
        (B.ssm_attn_decode if decode else B.ssm_attn_prefill)(ad, q, meta, pool, o, ws)
        B.ssm_gemm_nt(o, wout, y)
        at = 0
        for i, f, e in parts:
            got[i][f:e] = y[at:at + e - f]
            mid.append((i, f, e, qkv[at:at + e - f].clone(), q[at:at + e - f].clone()))
            at += e - f
    call([(0, 0, 20)], False)
    call([(0, 20, 40), (1, 0, 41)], False)
    call([(1, 41, 65)], False)
    for t in range(5):
        call([(0, 40 + t, 41 + t), (1, 65 + t, 66 + t)], True)
    assert B.take_status(ws) == 0
    for i, n in enumerate(lens):
        qkv, q = np.zeros((n, W)), np.zeros((n, hq, D))
        for j, f, e, m, qq in mid:
            if j == i:
                qkv[f:e], q[f:e] = _f64(m), _f64(qq).reshape(-1, hq, D)
        qo, ko, vo = oa.append(qkv, hq, hkv, range(n), qw.cpu().double().numpy(), kw.cpu().double().numpy(), 1e-5, rad, False)
        if fmt != "act":
            (ko, sk), (vo, sv) = oa.quantise(ko, fmt), oa.quantise(vo, fmt)
            ko, vo = ko * sk[..., None], vo * sv[..., None]
        o, _, _ = oa.attend(qo, ko, vo, range(n), ad.scale)
        want = o.reshape(n, hq * D) @ _f64(wout).T
        err = np.linalg.norm(_f64(got[i]) - want) / np.linalg.norm(want)
        # bf16: q, k, v (2^-8 each on scores and values), p, o and y rounded: well below six half steps;
        # 8 bits: a code that falls to the other side of a tie changes one value by 2^-4
        assert err < (6 * 2 ** -8 if act == "bf16" else 1e-5) + (2 ** -7 if fmt != "act" else 0), err
