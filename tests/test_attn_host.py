"""Paged attention cache without a GPU: the oracle against closed forms, and every refusal of the C entry
points (all checks are on the host, in front of the first launch)."""
import ctypes

import numpy as np
import pytest

from oracle import attention as oa
from paper_2602_21144_amd import binding as B


def _desc(**kw):
    d = dict(q_heads=8, kv_heads=2, head_dim=64, page_size=16, kv_format=0, act_dtype=B.SSM_BF16, window=0, scale=0.125)
    d.update(kw)
    return B.AttnDesc(**d)


def _rc(name, *args):
    return getattr(B.lib(), name)(*args)


# ------------------------------------------------------------------- oracle
def test_oracle_equal_scores_average_and_windows():
    k = np.zeros((5, 1, 4))
    v = np.arange(20.0).reshape(5, 1, 4)
    o, ab, _ = oa.attend(np.ones((1, 2, 4)), k, v, [4], 1.0)
    assert np.allclose(o, v.mean(0)) and np.allclose(ab, o)
    o, _, _ = oa.attend(np.ones((1, 2, 4)), k, v, [4], 1.0, window=2)
    assert np.allclose(o, v[3:5].mean(0))
    o, _, _ = oa.attend(np.ones((3, 2, 4)), k, v, [0, 1, 2], 1.0)
    assert np.allclose(o[0], v[0]) and np.allclose(o[2], v[:3].mean(0))
    o, _, _ = oa.attend(np.ones((1, 2, 4)), k, v, [4], 1.0, ok=np.zeros(5, bool))
    assert (o == 0).all()


def test_oracle_rotation_keeps_norms_and_relative_angles():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 8))
    rad = 10000.0 ** (-np.arange(4) / 4.0)
    for inter in (False, True):
        a = oa.rotate(q, 7, rad, inter) @ oa.rotate(k, 4, rad, inter)
        b = oa.rotate(q, 1003, rad, inter) @ oa.rotate(k, 1000, rad, inter)
        assert abs(a - b) < 1e-10
        assert abs(np.linalg.norm(oa.rotate(q, 12345, rad, inter)) - np.linalg.norm(q)) < 1e-12


def test_oracle_codes():
    v = oa.decode_codes(np.arange(256, dtype=np.uint8), "fp8")
    fin = v[np.isfinite(v)]
    assert fin.max() == 448 and np.isnan(v[127]) and np.isnan(v[255])
    assert np.array_equal(oa.round_e4m3(fin), fin)
    s = np.sort(np.unique(fin))
    x = np.random.default_rng(1).uniform(-448, 448, 2000)
    near = s[np.abs(x[:, None] - s[None]).argmin(1)]
    assert np.array_equal(oa.round_e4m3(x), near)
    c, sc = oa.quantise(np.array([[0.0, 0.0], [1.0, -2.0], [1e-31, 0.0]]), "int8")
    assert (c[0] == 0).all() and sc[0] == 0 and np.array_equal(c[1], [64, -127]) and sc[2] == 0


def test_rope_turns():
    rad = np.array([1.0, 1e-4, 0.0, -0.5, 2 * np.pi, 100.0])
    out = np.zeros(6, np.uint64)
    assert _rc("ssm_rope_turns", rad.ctypes.data, 6, out.ctypes.data) == 0
    got = out.astype(np.longdouble) / np.longdouble(2) ** 64
    want = np.mod(rad.astype(np.longdouble) / np.longdouble("6.283185307179586476925286766559"), 1)
    d = np.abs(got - want)
    assert (np.minimum(d, 1 - d) < 2.0 ** -60).all()
    # far positions: the wrapped product is the angle
    pos = np.uint64((1 << 30) - 1)
    ang = float(np.uint64(int(out[0]) * int(pos) % 2 ** 64).astype(np.longdouble) / np.longdouble(2) ** 64) * 2 * np.pi
    ref = float(np.fmod(np.longdouble(int(pos)), np.longdouble("6.283185307179586476925286766559")))
    assert abs(ang - ref) < 1e-8
    rad[2] = np.inf
    assert _rc("ssm_rope_turns", rad.ctypes.data, 6, out.ctypes.data) == B.SSM_E_INVAL
    assert _rc("ssm_rope_turns", None, 1, out.ctypes.data) == B.SSM_E_INVAL
    assert _rc("ssm_rope_turns", rad.ctypes.data, -1, out.ctypes.data) == B.SSM_E_INVAL
    assert _rc("ssm_rope_turns", None, 0, None) == 0


# ------------------------------------------------------------------- refusals
@pytest.mark.parametrize("kw", [dict(q_heads=0), dict(q_heads=7), dict(q_heads=256, kv_heads=2), dict(kv_heads=0), dict(kv_heads=16),
                                dict(head_dim=0), dict(head_dim=24), dict(head_dim=272), dict(page_size=8), dict(page_size=48),
                                dict(page_size=8192), dict(kv_format=3), dict(kv_format=-1), dict(act_dtype=2), dict(window=-1),
                                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_descriptor_refusals(kw):
    assert _rc("ssm_attn_check_desc", ctypes.byref(_desc(**kw))) == B.SSM_E_INVAL
    assert B.lib().ssm_last_error()
    n = ctypes.c_size_t()
    assert _rc("ssm_attn_workspace_bytes", ctypes.byref(_desc(**kw)), 1, 1, ctypes.byref(n)) == B.SSM_E_INVAL


def test_descriptor_accepts_the_range():
    assert _rc("ssm_attn_check_desc", None) == B.SSM_E_INVAL
    for hq, hkv in ((1, 1), (128, 1), (128, 128), (20, 4)):
        for d in range(16, 257, 16):
            for fmt in (0, 1, 2):
                for act in (B.SSM_F32, B.SSM_BF16):
                    assert _rc("ssm_attn_check_desc", ctypes.byref(_desc(q_heads=hq, kv_heads=hkv, head_dim=d, kv_format=fmt,
                                                                         act_dtype=act, window=5))) == 0


def test_workspace_grows_with_rows_and_sequences():
    for d in (_desc(), _desc(act_dtype=B.SSM_F32, head_dim=80), _desc(q_heads=128, kv_heads=1)):
        last = 0
        for t in (0, 1, 17, 300, 5000, 100000):
            n = B.attn_workspace_bytes(d, t, 4)
            assert n >= last and n >= 256
            last = n
        assert B.attn_workspace_bytes(d, 300, 9) >= B.attn_workspace_bytes(d, 300, 4)
    n = ctypes.c_size_t()
    d = ctypes.byref(_desc())
    for args in ((-1, 1, ctypes.byref(n)), (1, -1, ctypes.byref(n)), (1, 1, None), (1 << 31, 1, ctypes.byref(n))):
        assert _rc("ssm_attn_workspace_bytes", d, *args) == B.SSM_E_INVAL


@pytest.mark.parametrize("q,kv", [(32, 8), (32, 1), (128, 128), (128, 1), (16, 16), (1, 1)])
@pytest.mark.parametrize("dim", [96, 112, 128, 160])
def test_workspace_for_more_rows_serves_fewer(q, kv, dim):
    """Also where the larger call is cut into taller tiles (65536 rows of query heads)."""
    for act in (B.SSM_BF16, B.SSM_F32):
        d = _desc(q_heads=q, kv_heads=kv, head_dim=dim, act_dtype=act)
        edge = 65536 // q
        sizes = [B.attn_workspace_bytes(d, t, n) for t in (1, edge // 2, edge - 1, edge, edge + 1, 2 * edge) for n in (1, 40)]
        for n in (0, 1):
            assert sizes[n::2] == sorted(sizes[n::2])


def _host_meta(cu, kv, table, T=None, num=10, desc=None):
    cu = None if cu is None else np.array(cu, np.int32)
    kv, table = np.array(kv, np.int32), np.array(table, np.int32)
    T = (len(kv) if cu is None else int(cu[-1])) if T is None else T
    return _rc("ssm_kv_check_meta_host", ctypes.byref(desc or _desc()), None if cu is None else cu.ctypes.data, kv.ctypes.data,
               table.ctypes.data, len(kv), table.shape[1] if table.ndim == 2 else 0, T, num)


def test_host_metadata_check():
    ok = [[0, 1, 2], [3, 4, 5]]
    assert _host_meta([0, 5, 9], [20, 40], ok) == 0
    assert _host_meta(None, [20, 0], ok) == 0
    assert _host_meta([0, 5, 5], [20, 0], ok) == 0
    for cu, kv, T in (([1, 5, 9], [20, 40], 9), ([0, 6, 5], [20, 40], 5), ([0, 5, 9], [20, 40], 8), ([0, 5, 9], [4, 40], 9),
                      ([0, 5, 9], [20, 49], 9), ([0, 5, 9], [20, -1], 9), (None, [20, -1], 2), (None, [20, 40], 3)):
        assert _host_meta(cu, kv, ok, T) == -5, (cu, kv, T)
    assert _host_meta([0, 5, 9], [20, 40], [[0, 1, 2], [3, 10, 5]]) == -4
    assert _host_meta([0, 5, 9], [20, 40], [[0, -1, 2], [3, 4, 5]]) == -4
    assert _host_meta([0, 5, 9], [20, 40], [[0, 1, 99], [3, 4, 5]]) == 0      # behind the length: not looked at
    assert _host_meta([0, 1, 2], [33, 40], [[0, 1, 2], [0, 1, 5]]) == 0       # a shared prefix that nobody writes
    assert _host_meta([0, 1, 2], [33, 40], [[0, 1, 2], [0, 1, 2]]) == -4      # both write page 2
    assert _host_meta([0, 1, 2], [20, 40], [[0, 1, 2], [0, 1, 5]]) == -4      # one writes what the other reads
    assert _host_meta([0, 1, 2], [40, 20], [[0, 1, 5], [0, 1, 2]]) == -4      # in the other order too
    assert _host_meta([0, 1], [40], [[0, 3, 3]]) == -4                        # a sequence's written page named twice
    assert _host_meta([0, 1], [5], np.zeros((1, 0))) == B.SSM_E_INVAL
    assert _host_meta([0, 1], [5], [[0]], num=0) == B.SSM_E_INVAL


class _Fake:
    """Addresses that look like device memory: the refusals come before anything is read."""
    A = 0x10000


def _call(name, desc=None, T=4, meta=None, pool=None, ws=_Fake.A, wsb=1 << 30, **kw):
    d = desc or _desc()
    m = B.KvMetaC(_Fake.A, _Fake.A, _Fake.A, 2, 4) if meta is None else meta
    p = B.KvPoolC(_Fake.A, _Fake.A, _Fake.A, _Fake.A, 8) if pool is None else pool
    mp = None if m == "null" else ctypes.byref(m)
    pp = None if p == "null" else ctypes.byref(p)
    dp = ctypes.byref(d)
    g = dict(x=_Fake.A, ldx=8 * 64, o=2 * _Fake.A, ldo=8 * 64, tr=None)
    if name == "ssm_kv_append":
        g["ldx"] = 12 * 64
    if name == "ssm_kv_read":
        g.update(ldx=2 * 64, ldo=2 * 64)
    g.update(kw)
    if name == "ssm_kv_append":
        tr = None if g["tr"] is None else ctypes.byref(g["tr"])
        return _rc(name, dp, tr, g["x"], g["ldx"], T, mp, pp, g["o"], g["ldo"], ws, wsb, None)
    if name == "ssm_kv_read":
        return _rc(name, dp, T, mp, pp, g["x"], g["ldx"], g["o"], g["ldo"], ws, wsb, None)
    if name == "ssm_attn_prefill":
        return _rc(name, dp, g["x"], g["ldx"], T, mp, pp, g["o"], g["ldo"], ws, wsb, None)
    return _rc(name, dp, g["x"], g["ldx"], mp, pp, g["o"], g["ldo"], ws, wsb, None)


ALL = ["ssm_kv_append", "ssm_kv_read", "ssm_attn_prefill", "ssm_attn_decode"]


@pytest.mark.parametrize("name", ALL)
def test_call_refusals(name):
    A = _Fake.A
    I, L, W, Q = B.SSM_E_INVAL, B.SSM_E_ALIGN, B.SSM_E_WORKSPACE, -5
    assert _call(name, desc=_desc(head_dim=20)) == I
    assert _call(name, meta="null") == I and _call(name, pool="null") == I
    assert _call(name, meta=B.KvMetaC(A, None, A, 2, 4)) == I and _call(name, meta=B.KvMetaC(A, A, None, 2, 4)) == I
    assert _call(name, meta=B.KvMetaC(A, A, A, -1, 4)) == I and _call(name, meta=B.KvMetaC(A, A, A, 2, 0)) == I
    assert _call(name, meta=B.KvMetaC(A, A, A, 2, (1 << 26) + 1)) == I
    if name != "ssm_attn_decode":
        assert _call(name, meta=B.KvMetaC(A, A, A, 0, 4)) == Q
        assert _call(name, meta=B.KvMetaC(None, A, A, 2, 4)) == Q     # one row per sequence: T is nseq
        assert _call(name, T=-1) == I
        assert _call(name, T=0) == 0
    assert _call(name, pool=B.KvPoolC(None, A, None, None, 8)) == I and _call(name, pool=B.KvPoolC(A, A, None, None, 0)) == I
    assert _call(name, pool=B.KvPoolC(A, A + 8, None, None, 8)) == L
    assert _call(name, desc=_desc(kv_format=1), pool=B.KvPoolC(A, A, None, A, 8)) == I
    assert _call(name, desc=_desc(kv_format=2), pool=B.KvPoolC(A, A, A, A + 4, 8)) == L
    assert _call(name, ws=None) == I and _call(name, ws=A + 8) == L and _call(name, wsb=255) == W
    assert _call(name, x=None) == I and _call(name, o=None) == I
    assert _call(name, x=A + 8) == L and _call(name, o=A + 8) == L
    low = {"ssm_kv_read": 2 * 64}.get(name, 8 * 64)
    assert _call(name, ldo=low - 8) == I and _call(name, ldo=low + 4) == L
    if name.startswith("ssm_attn"):
        assert _call(name, o=A) == I
        assert _call(name, wsb=4096) == W
    assert B.lib().ssm_last_error()


@pytest.mark.parametrize("name", ALL)
def test_calls_larger_than_a_launch_are_refused(name):
    A, I = _Fake.A, B.SSM_E_INVAL
    assert _call(name, T=(1 << 15) + 1, meta=B.KvMetaC(A, A, A, (1 << 15) + 1, 4)) == I
    if name != "ssm_attn_decode":
        assert _call(name, T=(1 << 22) + 1, wsb=1 << 40) == I
        assert _call(name, T=1 << 31, wsb=1 << 40) == I
    n = ctypes.c_size_t()
    size = lambda t, s: _rc("ssm_attn_workspace_bytes", ctypes.byref(_desc(q_heads=128, kv_heads=128)), t, s, ctypes.byref(n))  # noqa: E731
    assert size((1 << 22) + 1, 1) == I and size(1, (1 << 15) + 1) == I
    assert size(1 << 22, 1 << 15) == 0 and n.value < 1 << 33


def test_host_check_of_a_pool_that_no_memory_describes():
    import resource
    used = int(open("/proc/self/statm").read().split()[0]) * resource.getpagesize()
    low, high = resource.getrlimit(resource.RLIMIT_AS)
    resource.setrlimit(resource.RLIMIT_AS, (used + (1 << 30), high))
    try:
        assert _host_meta([0, 5], [20], [[0, 1, 2]], num=(1 << 31) - 1) == B.SSM_E_INVAL
    finally:
        resource.setrlimit(resource.RLIMIT_AS, (low, high))
    assert _host_meta([0, 5], [20], [[0, 1, 2]]) == 0


def test_append_refusals():
    A = _Fake.A
    tr = lambda **kw: B.QkTransformC(**{**dict(q_norm_w=A, k_norm_w=A, turns=A, norm_eps=1e-5, rot_dim=32, interleaved=0), **kw})  # noqa: E731
    I, L = B.SSM_E_INVAL, B.SSM_E_ALIGN
    for bad in (dict(rot_dim=-8), dict(rot_dim=12), dict(rot_dim=72), dict(interleaved=2), dict(turns=None), dict(norm_eps=-1.0),
                dict(norm_eps=float("nan"))):
        assert _call("ssm_kv_append", tr=tr(**bad)) == I, bad
    for bad in (dict(turns=A + 8), dict(q_norm_w=A + 4), dict(k_norm_w=A + 8)):
        assert _call("ssm_kv_append", tr=tr(**bad)) == L, bad
    assert _call("ssm_kv_append", o=A, ldo=8 * 64) == I        # in place with another stride


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    ad = B.make_attn_desc(4, 2, 32, 16)
    with pytest.raises(B.SsmError):
        B.make_attn_desc(4, 3, 32, 16)
    with pytest.raises(KeyError):
        B.make_attn_desc(4, 2, 32, 16, kv_format="fp4")
    k = torch.zeros(3, 2, 16, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.KvPool(ad, k.float(), k)
    with pytest.raises(ValueError):
        B.KvPool(ad, k, k[:, :, :8])
    with pytest.raises(ValueError):
        B.KvPool(ad, k, k, torch.zeros(3, 2, 16), torch.zeros(3, 2, 16))
    with pytest.raises(ValueError):
        B.KvPool(ad, k, k)                       # host memory
    with pytest.raises(B.SsmError):
        B.KvMeta(ad, [0, 3], [2], [[0]], 4, device="cpu")
    with pytest.raises(ValueError):
        B.KvMeta(ad, [0, 3, 4], [3], [[0]], 4, device="cpu")
    m = B.KvMeta(ad, None, [3, 0], [[0], [1]], 4, device="cpu")
    assert m.T == 2 and m.cu is None and m.max_pages == 1
    with pytest.raises(ValueError):
        B.QkTransform(ad, torch.ones(16), None, device="cpu")
