"""Refusals of the paged attention cache's calls beyond those of single arguments, without a GPU."""
import ctypes

import numpy as np
import pytest

from paper_2602_21144_amd import binding as B

torch = pytest.importorskip("torch")


def _host_pool(ad, pages=3, heads=2, page=16, dim=32, dtype=torch.bfloat16, scales=False):
    """A pool over host memory: it never reaches a call."""
    p = object.__new__(B.KvPool)
    p.k, p.v = (torch.zeros(pages, heads, page, dim).to(dtype) for _ in range(2))
    p.k_scale, p.v_scale = (torch.zeros(pages, heads, page) if scales else None for _ in range(2))
    p.num_pages = pages
    p.check(ad)
    return p


CALLS = [lambda ad, m, p, x: B._m_ssm_kv_append(ad, None, x, m, p, x, x), lambda ad, m, p, x: B._m_ssm_kv_read(ad, m, p, x, x, x),
         lambda ad, m, p, x: B._m_ssm_attn_prefill(ad, x, m, p, x, x), lambda ad, m, p, x: B._m_ssm_attn_decode(ad, x, m, p, x, x)]


@pytest.mark.parametrize("call", CALLS)
def test_pool_or_meta_of_another_descriptor(call):
    """A call indexes by its own descriptor: a pool with smaller pages, fewer heads or narrower rows would be left behind."""
    ad = B.make_attn_desc(4, 2, 32, 16)
    pool, meta = _host_pool(ad), B.KvMeta(ad, None, [3], [[0]], 3, device="cpu")
    x = torch.zeros(1, 8 * 32, dtype=torch.bfloat16)
    for other in (B.make_attn_desc(4, 4, 32, 16), B.make_attn_desc(4, 2, 64, 16), B.make_attn_desc(4, 2, 32, 32),
                  B.make_attn_desc(4, 2, 32, 16, act="f32"), B.make_attn_desc(4, 2, 32, 16, kv_format="fp8"),
                  B.make_attn_desc(4, 1, 32, 16)):
        with pytest.raises(ValueError, match="expected"):
            call(other, meta, pool, x)
    wide = B.make_attn_desc(4, 2, 32, 32)
    with pytest.raises(ValueError, match="pages of 16 tokens"):
        call(wide, meta, _host_pool(wide, page=32), x)
    ad8 = B.make_attn_desc(4, 2, 32, 16, kv_format="int8")
    pool8 = _host_pool(ad8, dtype=torch.int8, scales=True)
    pool8.v_scale = torch.zeros(2, 2, 16)
    with pytest.raises(ValueError, match="v_scale"):
        call(ad8, meta, pool8, x)


def test_transform_of_another_descriptor():
    ad = B.make_attn_desc(4, 2, 32, 16)
    tr = object.__new__(B.QkTransform)
    tr.q_norm_w, tr.k_norm_w = torch.ones(16), None
    x = torch.zeros(1, 8 * 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="norm weight"):
        B._m_ssm_kv_append(ad, tr, x, B.KvMeta(ad, None, [3], [[0]], 3, device="cpu"), _host_pool(ad), x, x)


def _meta_rc(cu, kv, table, num, **desc):
    ad = B.AttnDesc(**{**dict(q_heads=8, kv_heads=2, head_dim=64, page_size=16, kv_format=0, act_dtype=B.SSM_BF16, window=0, scale=0.125),
                       **desc})
    cu = None if cu is None else np.array(cu, np.int32)
    kv, table = np.array(kv, np.int32), np.array(table, np.int32)
    T = len(kv) if cu is None else int(cu[-1])
    return B.lib().ssm_kv_check_meta_host(ctypes.byref(ad), None if cu is None else cu.ctypes.data, kv.ctypes.data, table.ctypes.data,
                                          len(kv), table.shape[1], T, num)


def test_host_check_of_pages_that_slid_out_of_the_window():
    slot = -4
    # 64 tokens, one row at 63: a window of 16 sees 48 .. 63, page 3 alone
    assert _meta_rc(None, [64], [[-1, -1, 9, 3]], 4, window=16) == 0
    assert _meta_rc(None, [64], [[-1, -1, 9, 3]], 4, window=17) == slot       # token 47 is on page 2
    assert _meta_rc(None, [64], [[-1, -1, 2, 3]], 4, window=17) == 0
    assert _meta_rc(None, [64], [[-1, -1, 2, 3]], 4) == slot                  # no window: all are seen
    # ten rows, the first at 54: a window of 16 sees from 39 on
    assert _meta_rc([0, 10], [64], [[-1, -1, 2, 3]], 4, window=16) == 0
    assert _meta_rc([0, 10], [64], [[-1, -1, -1, 3]], 4, window=16) == slot
    # a page that the first sequence gave back is written by the second, in either order
    assert _meta_rc(None, [64, 5], [[0, 1, 2, 3], [0, 0, 0, 0]], 4, window=20) == 0
    assert _meta_rc(None, [5, 64], [[0, 0, 0, 0], [0, 1, 2, 3]], 4, window=20) == 0
    assert _meta_rc(None, [64, 5], [[0, 1, 2, 3], [2, 0, 0, 0]], 4, window=20) == slot
    # the sequence's own first page again as its last
    assert _meta_rc(None, [64], [[3, 1, 2, 3]], 4, window=20) == 0 and _meta_rc(None, [64], [[3, 1, 2, 3]], 4) == slot
    # windows up to the largest, and one that nothing has slid out of
    assert _meta_rc(None, [64], [[0, 1, 2, 3]], 4, window=2 ** 31 - 1) == 0
    assert _meta_rc(None, [64], [[-1, 1, 2, 3]], 4, window=2 ** 31 - 1) == slot
    assert _meta_rc(None, [64], [[-1, 1, 2, 3]], 4, window=49) == slot and _meta_rc(None, [64], [[-1, 1, 2, 3]], 4, window=48) == 0
    # rows longer than the window: every page that they are on is written
    assert _meta_rc([0, 60], [64], [[-1, 1, 2, 3]], 4, window=4) == slot
    # a sequence without rows in the call: what its next one sees
    assert _meta_rc([0, 0], [64], [[-1, -1, -1, 3]], 4, window=17) == 0
    assert _meta_rc([0, 0], [64], [[-1, -1, -1, 3]], 4, window=18) == slot


A = 0x1000000   # looks like device memory: the refusals come before anything is read


def _op(name, x, ldx, o, ldo, T=4, act=B.SSM_BF16):
    """8 query heads and 2 kv heads of 64: rows of 768 (append), 128 (read) or 512 values into 512, 128 or 512."""
    d = ctypes.byref(B.AttnDesc(8, 2, 64, 16, 0, act, 0, 0.125))
    m = ctypes.byref(B.KvMetaC(A, A, A, T, 4))
    p = ctypes.byref(B.KvPoolC(A, A, None, None, 8))
    f = getattr(B.lib(), name)
    ws = (A, 1 << 40, None)
    if name == "ssm_kv_append":
        return f(d, None, x, ldx, T, m, p, o, ldo, *ws)
    if name == "ssm_kv_read":
        return f(d, T, m, p, x, ldx, o, ldo, *ws)
    if name == "ssm_attn_prefill":
        return f(d, x, ldx, T, m, p, o, ldo, *ws)
    return f(d, x, ldx, m, p, o, ldo, *ws)


WIDE = {"ssm_kv_append": (768, 512), "ssm_kv_read": (128, 128), "ssm_attn_prefill": (512, 512), "ssm_attn_decode": (512, 512)}


@pytest.mark.parametrize("name", list(WIDE))
@pytest.mark.parametrize("act,size", [(B.SSM_BF16, 2), (B.SSM_F32, 4)])
def test_operands_that_share_memory(name, act, size):
    wx, wo = WIDE[name]
    ld = wx + wo
    cases = [(A + 16, wx, wo), (A + 16, ld, ld), (A + (wx - 8) * size, ld, ld), (A - 16, ld, ld), (A - (wo - 8) * size, ld, ld),
             (A + 2 * ld * size, ld, ld), (A - 3 * ld * size, ld, ld), (A + (3 * ld + wx - 8) * size, ld, ld),
             (A - (3 * ld + wo - 8) * size, ld, ld), (A + ((wx - 8) + 3 * wx) * size, wx, wo), (A, wx + 8, wo),
             (A + (ld - 8) * size, ld, ld)]   # the last: its row ends in the next row's beginning
    if name != "ssm_kv_append":
        cases.append((A, ld, ld))
    for o, ldx, ldo in cases:
        assert _op(name, A, ldx, o, ldo, act=act) == B.SSM_E_INVAL, (hex(o), ldx, ldo)
        assert b"overlap" in B.lib().ssm_last_error() or o == A
    # strides that no memory holds
    assert _op(name, A, 1 << 60, A + 16, 1 << 60, act=act) == B.SSM_E_INVAL
    assert _op(name, A, ld, A + (wx - 8) * size, ld, T=1, act=act) == B.SSM_E_INVAL


def test_scales_up_to_the_largest_that_stays_finite():
    rc = lambda x: B.lib().ssm_attn_check_desc(ctypes.byref(B.AttnDesc(8, 2, 64, 16, 0, B.SSM_BF16, 0, x)))  # noqa: E731
    assert rc(2.3e38) == 0 and rc(1e-45) == 0
    assert rc(2.4e38) == B.SSM_E_INVAL and rc(3.4e38) == B.SSM_E_INVAL     # times log2(e): infinite


def test_metadata_that_32_bits_do_not_hold():
    ad = B.make_attn_desc(4, 2, 32, 16)
    big = 1 << 32
    for cu, kv, table in ((None, [3 + big], [[0]]), (None, [3], [[big]]), ([0, 3 + big], [3], [[0]]), (None, [2.5], [[0]])):
        for wrap in (np.array, torch.tensor):
            with pytest.raises(ValueError, match="32-bit"):
                B.KvMeta(ad, None if cu is None else wrap(cu), wrap(kv), wrap(table), 4, device="cpu")
    m = B.KvMeta(ad, torch.tensor([0, 3]), torch.tensor([20]), torch.tensor([[0, 2]]), 4, device="cpu")
    assert m.kv_len.dtype == torch.int32 and m.kv_len.tolist() == [20] and m.T == 3
    assert B.KvMeta(ad, None, [], [], 4, device="cpu").nseq == 0
