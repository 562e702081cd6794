"""The gated delta rule and its norms without a GPU: the oracle against closed forms, and every refusal of the C entry
points (all checks are on the host, in front of the first launch)."""
import ctypes

import numpy as np
import pytest

from delta_cases import Layer
from oracle import delta as od
from paper_2602_21144_amd import binding as B

torch = pytest.importorskip("torch")


def _rc(name, *args):
    return getattr(B.lib(), name)(*args)


# ------------------------------------------------------------------- oracle
def test_oracle_writes_and_reads_orthogonal_keys():
    """Orthogonal keys, no decay, full strength: a query of one key reads the value stored under it, and storing again
    replaces it."""
    dk = dv = 4
    qkv = np.zeros((3, 12))
    v = np.arange(12.0).reshape(3, 4) + 1
    for t, key in enumerate((0, 1, 0)):
        qkv[t, key] = qkv[t, 4 + key] = 1.0
        qkv[t, 8:] = v[t]
    o, pool, _ = od.run(qkv, np.full((3, 1), -800.0), np.full((3, 1), 800.0), [0.0], [0.0], [0, 3], [0], [0], np.zeros((1, 1, dv, dk)),
                        1, 1, dk, dv, qk_norm=False, scale=1.0)
    assert np.allclose(o[:, 0], v)
    assert np.allclose(pool[0, 0].T[:2], [v[2], v[1]]) and (pool[0, 0].T[2:] == 0).all()


def test_oracle_decay_and_strength():
    qkv = np.array([[1.0, 1.0, 2.0]] * 4)
    a = np.full((4, 1), np.log(np.expm1(0.5)))
    o, pool, _ = od.run(qkv, a, np.zeros((4, 1)), [0.0], [0.0], [0, 4], [0], [1], np.full((1, 1, 1, 1), 3.0), 1, 1, 1, 1, qk_norm=False,
                        scale=1.0)
    s, want = 3.0, []
    for _ in range(4):
        s = np.exp(-0.5) * s
        s += 0.5 * (2.0 - s)
        want.append(s)
    assert np.allclose(o[:, 0, 0], want) and np.allclose(pool, want[-1])


def test_oracle_chunk_form():
    """The rule of a chunk at once: U = (I + A)^-1 (beta V - beta e^G K S^T)."""
    L = Layer(torch, (1, 1, 16, 16), [40], "f32", seed=1, init=[1], beta_max=2.0)
    o, pool, _ = L.oracle()
    q, k, v = (x[:, 0] for x in od.split(L.qkv, 1, 1, 16, 16))
    q, k = (x / np.sqrt((x * x).sum(-1, keepdims=True) + 1e-6) for x in (q, k))
    _, b, a = L.columns(L.proj.astype(np.float64))
    G = np.cumsum(-np.exp(L.A_log.astype(np.float64)) * od.softplus(a[:, 0] + L.dt_bias))
    beta = 2.0 * od.sigmoid(b)
    D = np.exp(np.minimum(G[:, None] - G[None], 0.0))
    S = L.pool[L.slots[0], 0].astype(np.float64)
    A = np.tril(beta * D * (k @ k.T), -1)
    U = np.linalg.solve(np.eye(40) + A, beta * v - beta * np.exp(G)[:, None] * (k @ S.T))
    O = np.exp(G)[:, None] * (q @ S.T) / 4.0 + np.tril(D * (q @ k.T)) / 4.0 @ U
    assert np.allclose(O, o[:, 0], atol=1e-12)
    assert np.allclose(np.exp(G[-1]) * S + (np.exp(G[-1] - G)[:, None] * U).T @ k, pool[L.slots[0], 0], atol=1e-12)


def test_oracle_norms():
    x = np.array([[[3.0, 4.0]]])
    assert np.allclose(od.head_norm(x, np.ones(2), None, 0.0), x / np.sqrt(12.5))
    assert np.allclose(od.head_norm(x, np.array([2.0, 1.0]), np.zeros_like(x), 0.0, "sigmoid"), [[[3, 2]]] / np.sqrt(12.5))
    assert np.allclose(od.head_norm(x, np.ones(2), x * 0 + 2, 0.0, "identity", True), x / np.sqrt(12.5))
    r, n = od.block_norm(np.ones((1, 2)), [np.array([[3.0, 4.0]])], np.ones(2), 0.0, post_w=np.ones(2), scale=2.0)
    assert np.allclose(r, 1 + 2 * np.array([[3, 4]]) / np.sqrt(12.5)) and np.allclose((n * n).mean(), 1)


# ------------------------------------------------------------------- refusals
def _desc(**kw):
    d = dict(qk_heads=2, v_heads=4, qk_dim=64, v_dim=64, act_dtype=B.SSM_BF16, qk_norm=1, scale=0.125, norm_eps=1e-6, beta_max=1.0)
    d.update(kw)
    return B.DeltaDesc(**d)


@pytest.mark.parametrize("kw", [dict(v_heads=0), dict(qk_heads=0), dict(qk_heads=3), dict(v_heads=130, qk_heads=1), dict(qk_heads=8),
                                dict(qk_dim=0), dict(qk_dim=24), dict(qk_dim=272), dict(v_dim=8), dict(v_dim=72), dict(v_dim=528),
                                dict(act_dtype=2), dict(qk_norm=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                                dict(scale=float("inf")), dict(norm_eps=0.0), dict(norm_eps=float("inf")), dict(norm_eps=-1.0),
                                dict(beta_max=0.0), dict(beta_max=2.5), dict(beta_max=float("nan"))])
def test_descriptor_refusals(kw):
    assert _rc("ssm_delta_check_desc", ctypes.byref(_desc(**kw))) == B.SSM_E_INVAL
    assert B.lib().ssm_last_error()
    n = ctypes.c_size_t()
    assert _rc("ssm_delta_workspace_bytes", ctypes.byref(_desc(**kw)), 1, 1, ctypes.byref(n)) == B.SSM_E_INVAL


def test_descriptor_accepts_the_range():
    assert _rc("ssm_delta_check_desc", None) == B.SSM_E_INVAL
    for hk, hv in ((1, 1), (1, 128), (128, 128), (4, 20)):
        for dk in range(16, 257, 16):
            for dv in (16, 48, 512):
                assert _rc("ssm_delta_check_desc", ctypes.byref(_desc(qk_heads=hk, v_heads=hv, qk_dim=dk, v_dim=dv))) == 0


def test_workspace_grows_with_rows_and_sequences():
    for d in (_desc(), _desc(act_dtype=B.SSM_F32, qk_dim=256, v_dim=512), _desc(qk_heads=1, v_heads=128)):
        sizes = [B.delta_workspace_bytes(d, t, n) for t in (0, 1, 64, 65, 1000, 1 << 22) for n in (0, 1, 9, 1 << 15)]
        assert min(sizes) >= 256
        for i in range(4):
            assert sizes[i::4] == sorted(sizes[i::4])
        for i in range(6):
            assert sizes[4 * i:4 * i + 4] == sorted(sizes[4 * i:4 * i + 4])
    n = ctypes.c_size_t()
    d = ctypes.byref(_desc())
    for args in ((-1, 1, ctypes.byref(n)), (1, -1, ctypes.byref(n)), (1, 1, None), ((1 << 22) + 1, 1, ctypes.byref(n)),
                 (1, (1 << 15) + 1, ctypes.byref(n))):
        assert _rc("ssm_delta_workspace_bytes", d, *args) == B.SSM_E_INVAL


M = 1 << 20   # addresses that nothing is read from: every call below fails its checks, or has no rows


def _call(kind="prefill", desc=None, rows=100, **kw):
    d = desc or _desc()
    o = dict(qkv=16 * M, ld_qkv=512, a=32 * M, b=32 * M + 8, ld_ab=8, pool=64 * M, slots=8, out=48 * M, ld_out=256, ws=128 * M,
             ws_bytes=1 << 40, A_log=M, dt_bias=M, nseq=2, cu=M, slot=M, init=M, norm=None)
    assert not set(kw) - set(o), kw
    o.update(kw)
    gates = ctypes.byref(B.DeltaGatesC(o["A_log"], o["dt_bias"]))
    head = (ctypes.byref(d), gates, o["qkv"], o["ld_qkv"], o["a"], o["b"], o["ld_ab"])
    tail = (o["out"], o["ld_out"], o["ws"], o["ws_bytes"], None)
    if kind == "prefill":
        m = B.SeqMetaC(o["cu"], o["slot"], o["init"], o["nseq"])
        return _rc("ssm_delta_prefill", *head, rows, ctypes.byref(m), o["pool"], o["slots"], *tail)
    norm = None if o["norm"] is None else ctypes.byref(B.GatedNormC(*o["norm"]))
    return _rc("ssm_delta_decode", *head, rows, o["slot"], o["pool"], o["slots"], norm, *tail)


BAD = [(dict(qkv=None), -1), (dict(qkv=16 * M + 8), -2), (dict(ld_qkv=508), -1), (dict(ld_qkv=(1 << 22) + 8), -1), (dict(ld_qkv=516), -2), (dict(a=None), -1),
       (dict(b=None), -1), (dict(a=32 * M + 1), -2), (dict(ld_ab=3), -1), (dict(pool=None), -1), (dict(pool=64 * M + 4), -2),
       (dict(slots=0), -1), (dict(out=None), -1), (dict(out=48 * M + 2), -2), (dict(ld_out=248), -1), (dict(ld_out=260), -2), (dict(ld_out=(1 << 22) + 8), -1),
       (dict(ws=None), -1), (dict(ws=128 * M + 8), -2), (dict(ws_bytes=255), -3), (dict(A_log=None), -1), (dict(dt_bias=M + 4), -2),
       (dict(out=16 * M), -1), (dict(out=16 * M + 512), -1), (dict(a=48 * M, b=48 * M + 8), -1), (dict(b=48 * M + 2), -1),
       (dict(pool=48 * M), -1), (dict(pool=16 * M), -1), (dict(out=64 * M + 8 * 65536 - 16), -1)]


@pytest.mark.parametrize("kind", ["prefill", "decode"])
@pytest.mark.parametrize("kw,rc", BAD, ids=str)
def test_call_refusals(kw, rc, kind):
    assert _call(kind, **kw) == rc, B.lib().ssm_last_error()
    assert B.lib().ssm_last_error()


def test_call_refusals_of_each_kind():
    for rows in (-1, (1 << 22) + 1):
        assert _call(rows=rows) == -1
    for rows in (-1, (1 << 15) + 1):
        assert _call("decode", rows=rows) == -1
    assert _call(nseq=-1) == -1 and _call(nseq=(1 << 15) + 1) == -1 and _call(nseq=0) == -5
    assert _call(cu=None) == -1 and _call(slot=None) == -1 and _call(init=None) == -1 and _call("decode", slot=None) == -1
    assert _call(desc=_desc(qk_dim=24)) == -1
    # no sequences and no rows: nothing to do, whatever the rows' pointers
    assert _call(rows=0, nseq=0, qkv=None, a=None, b=None, out=None, cu=None, slot=None, init=None) == 0
    assert _call("decode", rows=0, qkv=None, a=None, b=None, out=None, slot=None) == 0
    w, z = M, 200 * M
    ok = (w, z, 256, 1e-5, 0, 2, 0)
    for bad, rc in ((dict(w=None), -1), (dict(w=M + 4), -2), (dict(z=z + 8), -2), (dict(ld=248), -1), (dict(ld=260), -2), (dict(eps=0.0), -1),
                    (dict(eps=float("nan")), -1), (dict(per_head=2), -1), (dict(gate=4), -1), (dict(gate=-1), -1), (dict(first=2), -1),
                    (dict(z=48 * M), -1)):
        n = dict(zip(("w", "z", "ld", "eps", "per_head", "gate", "first"), ok))
        n.update(bad)
        assert _call("decode", norm=tuple(n.values())) == rc, bad


def test_prefill_workspace_refusal():
    d = _desc()
    need = B.delta_workspace_bytes(d, 100, 2)
    assert _call(desc=d, ws_bytes=need - 1) == B.SSM_E_WORKSPACE


def _gated(x=M * 16, ld_x=256, dtype=1, T=10, heads=4, dim=64, norm=(M, M * 32, 256, 1e-5, 0, 2, 0), out=M * 48, ld_out=256):
    return _rc("ssm_gated_rmsnorm", x, ld_x, dtype, T, heads, dim, None if norm is None else ctypes.byref(B.GatedNormC(*norm)), out, ld_out, None)


def test_gated_norm_refusals():
    for kw, rc in ((dict(x=None), -1), (dict(x=16 * M + 2), -2), (dict(ld_x=248), -1), (dict(ld_x=252), -1), (dict(ld_x=260), -2),
                   (dict(dtype=2), -1), (dict(T=-1), -1), (dict(T=(1 << 22) + 1), -1), (dict(heads=0), -1), (dict(heads=513), -1),
                   (dict(dim=0), -1), (dict(dim=12), -1), (dict(dim=2056), -1), (dict(norm=None), -1), (dict(out=None), -1),
                   (dict(out=48 * M + 8), -2), (dict(ld_out=264, out=16 * M), -1), (dict(out=16 * M + 16), -1), (dict(out=32 * M), -1),
                   (dict(norm=(None, M * 32, 256, 1e-5, 0, 2, 0)), -1), (dict(norm=(M, M * 32, 256, 0.0, 0, 2, 0)), -1)):
        assert _gated(**kw) == rc, kw
    assert _gated(T=0, x=None, out=None) == 0


def _block(base=M * 16, bdt=0, parts=(M * 32,), n=None, pdt=1, blk=(None, None, 0, 0.0, 1.0, 0, 0), res=M * 48, w=M, eps=1e-5,
           normed=M * 64, ndt=1, T=10, d=256):
    arr = (ctypes.c_void_p * 9)(*parts) if parts is not None else None
    n = len(parts) if n is None and parts is not None else n
    return _rc("ssm_block_rmsnorm", base, bdt, arr, n, pdt, None if blk is None else ctypes.byref(B.BlockOutC(*blk)), res, w, eps, normed, ndt,
               T, d, None)


def test_block_norm_refusals():
    nan = float("nan")
    for kw, rc in ((dict(base=None), -1), (dict(base=16 * M + 4), -2), (dict(bdt=2), -1), (dict(pdt=5), -1), (dict(ndt=-1), -1),
                   (dict(parts=(None,)), -1), (dict(parts=(32 * M + 2,)), -2), (dict(parts=None, n=1), -1), (dict(n=9), -1), (dict(n=-1), -1),
                   (dict(blk=None), -1), (dict(blk=(M, None, 0, 0.0, 1.0, 0, 0)), -1), (dict(blk=(M + 4, None, 0, 1e-5, 1.0, 0, 0)), -2),
                   (dict(blk=(None, None, 0, 0.0, nan, 0, 0)), -1), (dict(blk=(None, None, 0, 0.0, 1.0, 0, 4)), -1),
                   (dict(blk=(None, 80 * M, 0, 0.0, 1.0, 3, 0)), -1), (dict(blk=(None, 80 * M, 248, 0.0, 1.0, 0, 0)), -1),
                   (dict(blk=(None, 80 * M, 260, 0.0, 1.0, 0, 0)), -2), (dict(blk=(None, 80 * M + 4, 0, 0.0, 1.0, 0, 0)), -2),
                   (dict(res=None), -1), (dict(w=None), -1), (dict(normed=None), -1), (dict(eps=0.0), -1), (dict(eps=nan), -1),
                   (dict(d=0), -1), (dict(d=12), -1), (dict(d=8200), -1), (dict(T=-1), -1), (dict(T=(1 << 22) + 1), -1),
                   (dict(base=48 * M + 16), -1), (dict(base=48 * M, bdt=1), -1), (dict(base=64 * M), -1), (dict(parts=(48 * M,)), -1),
                   (dict(parts=(64 * M + 16,)), -1), (dict(normed=48 * M), -1), (dict(blk=(None, 64 * M, 0, 0.0, 1.0, 0, 0)), -1),
                   (dict(blk=(None, 48 * M - 16, 0, 0.0, 1.0, 0, 0)), -1)):
        assert _block(**kw) == rc, kw
    assert _block(T=0, base=None, res=None, normed=None, w=None) == 0


def test_binding_refuses_other_shapes():
    dd = B.make_delta_desc(2, 4, 64, 64)
    cpu = torch.zeros(4)
    with pytest.raises(ValueError):
        B.DeltaGates(dd, torch.zeros(3), cpu)
    with pytest.raises(ValueError):
        B.GatedNorm(torch.zeros(65), None, 4, 64)
    with pytest.raises(B.SsmError):
        B.make_delta_desc(3, 4, 64, 64)
