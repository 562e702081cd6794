"""The gated delta rule on the GPU against the float64 oracle: prompts, single tokens, the two together, and the edges
of what the calls accept."""
import numpy as np
import pytest

from delta_cases import Layer, f64, near, out_bound, state_bound
from oracle import delta as od

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _prefill(L, rows_behind=0, ws_for=None, strided=False, meta=None, stream=None, num_slots=None):
    """One call with poisoned outputs: (out, pool, status, rows behind the last sequence)."""
    from paper_2602_21144_amd import binding as B
    dd = L.desc(B)
    T = L.T + rows_behind
    pad = lambda x: np.concatenate([x, np.full((rows_behind, x.shape[1]), np.nan, np.float32)])  # noqa: E731
    qkv, proj = L.dev(pad(L.qkv)), L.dev(pad(L.proj))
    if strided:
        wide = torch.full((T, qkv.shape[1] + 24), float("nan"), dtype=qkv.dtype, device="cuda")
        wide[:, 8:8 + qkv.shape[1]] = qkv
        qkv = wide[:, 8:8 + qkv.shape[1]]
    out = torch.full((T, L.wide + (16 if strided else 0)), float("nan"), dtype=L.tdt, device="cuda")
    pool = L.dev(L.pool, False)
    meta = meta or B.SeqMeta(L.cu, L.slots, L.init, L.S)
    meta.T = T
    ws = B.workspace(B.delta_workspace_bytes(dd, *(ws_for or (T, L.n))))
    _, b, a = L.columns(proj)
    if stream is not None:
        torch.cuda.synchronize()
    B.ssm_delta_prefill(dd, L.gates(B, dd), qkv, a, b, meta, pool, out[:, :L.wide], ws, stream=stream)
    torch.cuda.synchronize()
    if strided:
        assert torch.isnan(out[:, L.wide:]).all()
        out = out[:, :L.wide].contiguous()
    return out, pool, B.take_status(ws), out[L.T:]


def _check(L, out, pool, what=""):
    o, want, sizes = L.oracle()
    near(f64(out[:L.T]).reshape(o.shape), o, out_bound(o, sizes, L.act), f"{what} out")
    got = f64(pool)
    near(got[L.slots], want[L.slots], state_bound(want[L.slots], L.act), f"{what} state")
    others = [s for s in range(L.S) if s not in L.slots]
    assert np.array_equal(got[others], L.pool[others].astype(np.float64)), f"{what}: a slot that no sequence names changed"


HEADS = [(1, 1, 16, 16), (2, 4, 64, 64), (1, 3, 80, 48), (2, 2, 128, 128), (2, 2, 96, 192), (1, 2, 112, 112), (1, 1, 144, 32),
         (1, 1, 256, 512), (1, 20, 32, 16)]
LENS = [[1], [64], [65], [63, 0, 130, 1], [2, 3, 128, 16, 17]]


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_prefill(heads, lens, act):
    L = Layer(torch, heads, lens, act, seed=len(lens) + heads[2])
    out, pool, status, behind = _prefill(L, rows_behind=3)
    assert status == 0 and torch.isnan(behind).all()
    _check(L, out, pool)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(qk_norm=False), dict(beta_max=2.0), dict(decay=300.0), dict(decay=1e-6, init=[1])], ids=str)
def test_prefill_forms(kw, act):
    L = Layer(torch, (2, 2, 64, 64), [333], act, seed=3, **kw)
    out, pool, status, _ = _prefill(L)
    assert status == 0
    _check(L, out, pool)


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_prefill_of_a_long_prompt(act):
    L = Layer(torch, (1, 1, 128, 128), [3001, 40], act, seed=4, init=[1, 0])
    out, pool, status, _ = _prefill(L, strided=True)
    assert status == 0
    _check(L, out, pool)


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_prefill_with_keys_that_repeat(act):
    """The same key again and again with beta near one: the sums of a chunk cancel as far as they can."""
    L = Layer(torch, (1, 2, 64, 64), [200], act, seed=5, beta_max=1.0, decay=1e-4)
    L.qkv[:, 64:128] = L.qkv[:1, 64:128]
    L.proj[:, L.wide:L.wide + 2] = L.stored(np.full((200, 2), 12.0))
    out, pool, _, _ = _prefill(L)
    _check(L, out, pool)


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_prefill_gates_at_their_ends(act):
    """Tokens that forget everything between tokens that forget nothing, and write strengths of 0 and 1: what follows a
    reset is as exact as without it."""
    L = Layer(torch, (1, 2, 64, 64), [150], act, seed=6, init=[1])
    L.A_log[:] = np.log(16.0)
    L.dt_bias[:] = 0.0
    a = L.proj[:, L.wide + 2:L.wide + 4]
    a[:] = -12.0
    a[[20, 85]] = 10000.0
    a[50] = -1000.0
    b = L.proj[:, L.wide:L.wide + 2]
    b[[10, 90]], b[[11, 91]] = -200.0, 200.0
    L.proj = L.stored(L.proj)
    out, pool, _, _ = _prefill(L)
    _check(L, out, pool)


def test_prefill_zero_rows_of_queries_and_keys():
    L = Layer(torch, (2, 2, 64, 64), [70], "bf16", seed=7)
    L.qkv[3:6, :256] = 0.0
    out, pool, _, _ = _prefill(L)
    _check(L, out, pool)


def test_prefill_many_short_sequences():
    rng = np.random.default_rng(8)
    L = Layer(torch, (1, 1, 32, 16), list(rng.integers(0, 5, 700)), "bf16", seed=8)
    out, pool, status, _ = _prefill(L)
    assert status == 0
    _check(L, out, pool)


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_prefill_in_pieces_is_the_whole(act):
    """A prompt in two calls, the second from the cached state, against the oracle of the whole prompt."""
    whole = Layer(torch, (2, 4, 128, 64), [301], act, seed=9, init=[0])
    o, want, sizes = whole.oracle()
    got, pool = [], whole.pool
    for lo, hi in ((0, 77), (77, 301)):
        part = Layer(torch, (2, 4, 128, 64), [hi - lo], act, seed=9, init=[int(lo > 0)])
        part.qkv, part.proj, part.A_log, part.dt_bias = whole.qkv[lo:hi], whole.proj[lo:hi], whole.A_log, whole.dt_bias
        part.pool, part.slots = pool, whole.slots
        out, p, _, _ = _prefill(part)
        got.append(f64(out))
        pool = f64(p).astype(np.float32)
    # the second piece begins inside a 64-token chunk of the whole: twice the sizes cover either cut
    near(np.concatenate(got).reshape(o.shape), o, out_bound(o, 2 * sizes, act), "out")
    near(pool[whole.slots], want[whole.slots], 2 * state_bound(want[whole.slots], act), "state")


def test_a_workspace_for_more_serves_fewer():
    L = Layer(torch, (2, 4, 64, 64), [100, 1, 29], "bf16", seed=10)
    out, pool, status, _ = _prefill(L, ws_for=(5000, 40))
    assert status == 0
    _check(L, out, pool)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("heads,lens", [((16, 32, 128, 128), [70, 1, 65]), ((32, 64, 64, 80), [66, 40]), ((20, 60, 96, 64), [3, 130, 1, 0, 64]),
                                        ((4, 12, 192, 192), [64, 100, 1, 70]), ((8, 8, 256, 512), [65, 3, 90]), ((64, 64, 32, 48), [20, 3, 65])],
                         ids=str)
def test_prefill_of_many_heads(heads, lens, act):
    """More pairs of a head and a sequence than run at once, by workgroups of four waves of columns; head counts that
    the eight XCDs do not divide, three value heads to a q/k head, columns that leave waves without any."""
    L = Layer(torch, heads, lens, act, seed=sum(heads), init=[i % 2 for i in range(len(lens))])
    out, pool, status, behind = _prefill(L, rows_behind=1)
    assert status == 0 and torch.isnan(behind).all()
    _check(L, out, pool)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("size", [2.0 ** -40, 1.0, 2.0 ** 30])
def test_prefill_far_scales(size, act):
    """Values and states far from one, and keys of the program's own lengths from 2^-12 to 1: what is scaled inside
    comes back."""
    L = Layer(torch, (1, 2, 64, 64), [150], act, seed=19, init=[1], qk_norm=False)
    L.qkv[:, 128:] *= size
    L.pool *= np.float32(size)
    L.qkv[:, 64:128] = L.stored(L.qkv[:, 64:128] * 2.0 ** -np.random.default_rng(1).integers(0, 13, (150, 1)))
    out, pool, _, _ = _prefill(L)
    _check(L, out, pool)


def test_runs_give_the_same_bits():
    L = Layer(torch, (2, 4, 128, 128), [257, 64, 500], "bf16", seed=11)
    a, b = _prefill(L), _prefill(L)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ------------------------------------------------------------------- device metadata
def test_bad_slots_and_lengths():
    from paper_2602_21144_amd import binding as B
    L = Layer(torch, (1, 2, 64, 64), [70, 30, 100], "bf16", seed=12, init=[1, 1, 0])
    meta = B.SeqMeta(L.cu, L.slots, L.init, L.S)
    meta.slot[1] = L.S
    out, pool, status, _ = _prefill(L, meta=meta)
    assert status == B.SSM_STATUS_BAD_SLOT
    init = L.init.copy()
    init[1] = 0
    o, want, sizes = L.oracle(init=init)
    near(f64(out).reshape(o.shape), o, out_bound(o, sizes, "bf16"), "out")   # from zeros, nothing stored
    want[L.slots[1]] = L.pool[L.slots[1]]
    near(f64(pool), want, state_bound(want, "bf16"), "state")
    assert np.array_equal(f64(pool)[L.slots[1]], L.pool[L.slots[1]].astype(np.float64))

    for bad in ([0, 70, 60, 200], [0, 70, 201, 200], [-5, 70, 100, 200], [0, 70, 2 ** 31 - 1, 200]):
        meta = B.SeqMeta(L.cu, L.slots, L.init, L.S)
        meta.cu.copy_(torch.tensor(bad, dtype=torch.int32))
        out, pool, status, _ = _prefill(L, meta=meta)
        assert status & B.SSM_STATUS_BAD_SEQLENS
        for i in range(3):   # a sequence whose own entries do not fit leaves its slot alone
            if bad[i] < 0 or bad[i + 1] < bad[i] or bad[i + 1] > L.T:
                assert np.array_equal(f64(pool)[L.slots[i]], L.pool[L.slots[i]].astype(np.float64))
            elif list(bad[i:i + 2]) == list(L.cu[i:i + 2]):
                o, want, sizes = L.oracle()
                lo, hi = L.cu[i], L.cu[i + 1]
                near(f64(pool)[L.slots[i]], want[L.slots[i]], state_bound(want[L.slots[i]], "bf16"), "state")
                if bad[1:3] != [70, 60]:   # there the third sequence begins inside the first
                    near(f64(out).reshape(o.shape)[lo:hi], o[lo:hi], out_bound(o, sizes, "bf16")[lo:hi], "out")


def test_overlapping_sequences_stay_inside_the_workspace():
    """Every second of many sequences names all rows of the call: far more chunks than a call of that many rows has."""
    from paper_2602_21144_amd import binding as B
    n, T = 64, 640
    L = Layer(torch, (1, 1, 32, 16), [T] + [0] * (n - 1), "bf16", seed=13)
    meta = B.SeqMeta(L.cu, L.slots, L.init, L.S)
    meta.cu.copy_(torch.tensor([0, T] * (n // 2) + [0], dtype=torch.int32))
    _, _, status, _ = _prefill(L, meta=meta)
    assert status & B.SSM_STATUS_BAD_SEQLENS


def test_empty_sequences():
    L = Layer(torch, (1, 2, 64, 64), [0, 5, 0], "bf16", seed=14, init=[0, 0, 1])
    out, pool, status, _ = _prefill(L)
    assert status == 0
    _check(L, out, pool)
    assert (f64(pool)[L.slots[0]] == 0).all() and np.array_equal(f64(pool)[L.slots[2]], L.pool[L.slots[2]])


@pytest.mark.parametrize("n", [2, 300])
@pytest.mark.parametrize("rows", [0, 5])
def test_call_without_tokens(n, rows):
    """Nothing but the states of fresh sequences is written, which become zeros."""
    L = Layer(torch, (1, 2, 64, 64), [0] * n, "f32", seed=16, init=[0, 1] * (n // 2))
    out, pool, status, behind = _prefill(L, rows_behind=rows)
    assert status == 0 and out.shape[0] == rows and torch.isnan(behind).all()
    want = L.pool.copy()
    want[L.slots[::2]] = 0
    assert np.array_equal(f64(pool), want, equal_nan=True)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_values_that_are_not_finite(act, value):
    """In v of one head, in a sequence between two others: nothing of another head or sequence and nothing more than 63
    rows in front changes; its own row and the state are not finite."""
    L = Layer(torch, (1, 2, 64, 64), [90, 200, 64], act, seed=15)
    o, want, sizes = L.oracle()
    at = 90 + 150
    L.qkv[at, 128 + 64 + 5] = value          # head 1, value 5
    out, pool, _, _ = _prefill(L)
    got = f64(out).reshape(o.shape)
    assert not np.isfinite(got[at, 1, 5])
    rows = np.r_[0:at - 63, 290:354]
    tol = out_bound(o, sizes, act)
    near(got[rows], o[rows], tol[rows], "rows of others")
    near(got[:, 0], o[:, 0], tol[:, 0], "the other head")
    st = f64(pool)
    assert not np.isfinite(st[L.slots[1], 1, 5]).any()
    near(st[L.slots][:, 0], want[L.slots][:, 0], state_bound(want[L.slots], act)[:, 0], "states of the other head")
    near(st[L.slots[[0, 2]]], want[L.slots[[0, 2]]], state_bound(want[L.slots[[0, 2]]], act), "states of the others")


# ------------------------------------------------------------------- single tokens
def _decode(L, norm=None, slots=None, stream=None):
    from paper_2602_21144_amd import binding as B
    dd = L.desc(B)
    qkv, proj, pool = L.dev(L.qkv), L.dev(L.proj), L.dev(L.pool, False)
    z, b, a = L.columns(proj)
    out = torch.full((L.n, L.wide), float("nan"), dtype=L.tdt, device="cuda")
    ws = B.workspace(B.delta_workspace_bytes(dd, L.n, L.n))
    gn = None
    if norm is not None:
        w, with_z, kw = norm
        gn = B.GatedNorm(L.dev(w, False), z if with_z else None, L.hv, L.dv, **kw)
    slot = torch.from_numpy(L.slots if slots is None else slots).cuda()
    B.ssm_delta_decode(dd, L.gates(B, dd), qkv, a, b, slot, pool, out, ws, norm=gn, stream=stream)
    torch.cuda.synchronize()
    return out, pool, B.take_status(ws)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [1, 5, 70])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_decode(heads, batch, act):
    if batch == 70 and heads[2] * heads[3] > 20000:
        pytest.skip("the oracle would take long, and smaller heads cover the batch")
    L = Layer(torch, heads, [1] * batch, act, seed=batch + heads[3], init=[1] * batch)
    out, pool, status = _decode(L)
    assert status == 0
    # float32 throughout: one rounding of the output, sums of at most 256 products
    o, want, sizes = L.oracle()
    half = 2.0 ** -8 if act == "bf16" else 2.0 ** -24
    near(f64(out).reshape(o.shape), o, half * np.abs(o) + 64 * 2.0 ** -24 * sizes + 1e-30, "out")
    near(f64(pool)[L.slots], want[L.slots], state_bound(want[L.slots], act), "state")
    others = [s for s in range(L.S) if s not in L.slots]
    assert np.array_equal(f64(pool)[others], L.pool[others].astype(np.float64))


def _norm_bound(o, sizes, y, w, z, act, kw):
    """The norm of o + d with |d| <= 64 2^-24 sizes: d / rms and o / rms times the relative error of the rms, which is at
    most rms(d) / rms; then the float32 of the norm itself (16 steps) and one rounding."""
    f = np.ones_like(o) if z is None else np.abs(od.gate(z, kw.get("gate", "silu")))
    d = 64 * 2.0 ** -24 * sizes
    first = kw.get("gate_first", False)
    x, d = (o * f, d * f) if first else (o, d)
    rms = np.sqrt((x * x).mean(-1, keepdims=True) + kw.get("eps", 1e-5))
    dy = (d + np.abs(x) * np.sqrt((d * d).mean(-1, keepdims=True)) / rms) / rms * np.abs(w) * (1 if first else f)
    return (2.0 ** -8 if act == "bf16" else 2.0 ** -24) * np.abs(y) + 16 * 2.0 ** -24 * np.abs(y) + dy + 1e-30


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [(2, 4, 128, 128), (1, 3, 80, 48), (1, 1, 256, 512)], ids=str)
@pytest.mark.parametrize("per_head,with_z,kw", [(False, True, {}), (True, True, dict(gate="sigmoid", gate_first=True, eps=1e-3)),
                                                (False, False, {}), (True, True, dict(gate="identity"))])
def test_decode_with_the_head_norm(heads, per_head, with_z, kw, act):
    L = Layer(torch, heads, [1] * 3, act, seed=21, init=[1] * 3)
    w = (1 + 0.1 * np.random.default_rng(1).standard_normal(L.wide if per_head else L.dv)).astype(np.float32)
    out, pool, status = _decode(L, (w, with_z, kw))
    assert status == 0
    o, want, sizes = L.oracle()
    z = L.columns(L.proj)[0].astype(np.float64).reshape(o.shape) if with_z else None
    wf = w.astype(np.float64).reshape(L.hv if per_head else 1, L.dv)
    y = od.head_norm(o, wf, z, kw.get("eps", 1e-5), kw.get("gate", "silu"), kw.get("gate_first", False))
    near(f64(out).reshape(o.shape), y, _norm_bound(o, sizes, y, wf, z, act, kw), "out")
    near(f64(pool)[L.slots], want[L.slots], state_bound(want[L.slots], act), "state")


def test_decode_of_states_that_no_cache_keeps():
    """More than 96 MB of states, which go past the caches."""
    n, heads = 50, (16, 32, 128, 128)
    L = Layer(torch, heads, [1] * n, "bf16", seed=24, init=[1] * n)
    out, pool, status = _decode(L)
    assert status == 0
    o, want, sizes = L.oracle()
    near(f64(out).reshape(o.shape), o, 2.0 ** -8 * np.abs(o) + 64 * 2.0 ** -24 * sizes + 1e-30, "out")
    near(f64(pool)[L.slots], want[L.slots], state_bound(want[L.slots], "bf16"), "state")


def test_decode_bad_slots():
    from paper_2602_21144_amd import binding as B
    L = Layer(torch, (1, 2, 64, 64), [1] * 4, "bf16", seed=22, init=[1] * 4)
    slots = L.slots.copy()
    slots[1], slots[3] = -1, L.S
    out, pool, status = _decode(L, slots=slots)
    assert status == B.SSM_STATUS_BAD_SLOT
    assert (f64(out)[[1, 3]] == 0).all()
    o, want, sizes = L.oracle()
    near(f64(out).reshape(o.shape)[[0, 2]], o[[0, 2]], out_bound(o, sizes, "bf16")[[0, 2]], "out")
    keep = [s for s in range(L.S) if s not in L.slots[[0, 2]]]
    assert np.array_equal(f64(pool)[keep], L.pool[keep].astype(np.float64))


def test_decode_states_behind_four_gigabytes():
    """A slot whose states lie behind 2^32 bytes and 2^31 values of the pool."""
    from paper_2602_21144_amd import binding as B
    hv, dv, dk = 32, 128, 128
    L = Layer(torch, (16, hv, dk, dv), [1], "bf16", seed=23, init=[1], spare=0)
    S = 2 ** 31 // (hv * dv * dk) + 3
    dd = L.desc(B)
    pool = torch.empty(S, hv, dv, dk, dtype=torch.float32, device="cuda")
    pool[S - 1] = L.dev(L.pool[0], False)
    pool[S - 2] = 7.0
    qkv, proj = L.dev(L.qkv), L.dev(L.proj)
    _, b, a = L.columns(proj)
    slot = torch.tensor([S - 1], dtype=torch.int32, device="cuda")
    ws = B.workspace(B.delta_workspace_bytes(dd, 1, 1))
    o, want, sizes = L.oracle()
    for kind in ("decode", "prefill"):
        pool[S - 1] = L.dev(L.pool[0], False)
        out = torch.empty(1, L.wide, dtype=L.tdt, device="cuda")
        if kind == "decode":
            B.ssm_delta_decode(dd, L.gates(B, dd), qkv, a, b, slot, pool, out, ws)
        else:
            B.ssm_delta_prefill(dd, L.gates(B, dd), qkv, a, b, B.SeqMeta([0, 1], [S - 1], [1], S), pool, out, ws)
        near(f64(out).reshape(o.shape), o, out_bound(o, sizes, "bf16"), f"{kind} out")
        near(f64(pool[S - 1])[None], want, state_bound(want, "bf16"), f"{kind} state")
        assert (pool[S - 2] == 7.0).all()
    assert B.take_status(ws) == 0


# ------------------------------------------------------------------- as they are used
@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_a_prompt_and_its_next_tokens(act):
    """A prompt, then token by token in place, against the oracle of the whole."""
    from paper_2602_21144_amd import binding as B
    heads, n, steps = (2, 4, 64, 64), 3, 6
    lens = [70, 1, 129]
    whole = Layer(torch, heads, [m + steps for m in lens], act, seed=31, init=[0, 1, 0])
    o, want, sizes = whole.oracle()
    prompt = [whole.cu[i] + t for i, m in enumerate(lens) for t in range(m)]
    L = Layer(torch, heads, lens, act, seed=31, init=[0, 1, 0])
    L.qkv, L.proj, L.pool, L.slots = whole.qkv[prompt], whole.proj[prompt], whole.pool, whole.slots
    L.A_log, L.dt_bias = whole.A_log, whole.dt_bias
    out, pool, _, _ = _prefill(L)
    near(f64(out).reshape(-1, 4, 64), o[prompt], out_bound(o, sizes, act)[prompt], "prompt")
    dd = L.desc(B)
    gates, ws, slot = L.gates(B, dd), B.workspace(B.delta_workspace_bytes(dd, n, n)), torch.from_numpy(L.slots).cuda()
    for s in range(steps):
        at = [whole.cu[i] + m + s for i, m in enumerate(lens)]
        qkv, proj = L.dev(whole.qkv[at]), L.dev(whole.proj[at])
        _, b, a = L.columns(proj)
        y = torch.empty(n, L.wide, dtype=L.tdt, device="cuda")
        B.ssm_delta_decode(dd, gates, qkv, a, b, slot, pool, y, ws)
        near(f64(y).reshape(-1, 4, 64), o[at], out_bound(o, 2 * sizes, act)[at], f"token {s}")
    near(f64(pool)[L.slots], want[L.slots], 2 * state_bound(want[L.slots], act), "state")


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_captured_steps_replay_like_eager(act):
    """A prompt and two decode steps with the head norm in one graph, replayed between eager work."""
    from paper_2602_21144_amd import binding as B
    L = Layer(torch, (2, 4, 64, 64), [150, 33], act, seed=41)
    dd = L.desc(B)
    gates = L.gates(B, dd)
    qkv, proj, pool0 = L.dev(L.qkv), L.dev(L.proj), L.dev(L.pool, False)
    z, b, a = L.columns(proj)
    pool, out, y = pool0.clone(), torch.empty(L.T, L.wide, dtype=L.tdt, device="cuda"), torch.empty(2, L.wide, dtype=L.tdt, device="cuda")
    slot = torch.from_numpy(L.slots).cuda()
    meta, ws = B.SeqMeta(L.cu, L.slots, L.init, L.S), B.workspace(B.delta_workspace_bytes(dd, L.T, L.n))
    w = torch.ones(L.dv, device="cuda")
    s = torch.cuda.Stream()
    calls = [B.bind("ssm_delta_prefill", dd, gates, qkv, a, b, meta, pool, out, ws, stream=s)]
    calls += [B.bind("ssm_delta_decode", dd, gates, qkv[r:r + 2], a[r:r + 2], b[r:r + 2], slot, pool, y, ws,
                     norm=B.GatedNorm(w, z[r:r + 2], L.hv, L.dv), stream=s) for r in (0, 2)]
    torch.cuda.synchronize()
    for c in calls:
        c()
    torch.cuda.synchronize()
    ref = [t.clone() for t in (out, y, pool)]
    pool.copy_(pool0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        for c in calls:
            c()
    torch.cuda.synchronize()
    for _ in range(3):
        pool.copy_(pool0)
        out.fill_(float("nan"))
        y.fill_(float("nan"))
        torch.randn(1000, device="cuda") @ torch.randn(1000, device="cuda")
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip((out, y, pool), ref):
            assert torch.equal(got, want)
    assert B.take_status(ws) == 0


def test_another_stream():
    L = Layer(torch, (2, 4, 128, 64), [300, 5], "bf16", seed=42)
    ref = _prefill(L)
    got = _prefill(L, stream=torch.cuda.Stream())
    assert torch.equal(ref[0], got[0]) and torch.equal(ref[1], got[1])


@pytest.mark.parametrize("act", ["bf16", "f32"])
def test_a_block_of_a_stack(act):
    """Projection, rule, head norm, projection back, and what lies between two blocks, as a layer runs them; every stage
    against the oracle of what the stage before it left."""
    from paper_2602_21144_amd import binding as B
    heads, d = (2, 4, 64, 64), 192
    L = Layer(torch, heads, [80, 21], act, seed=43, init=[0, 1])
    rng = np.random.default_rng(44)
    wide, rows = L.wide, 2 * 2 * 64 + 2 * L.wide + 8
    w_in, w_out = L.stored(rng.standard_normal((rows, d)) / d ** 0.5), L.stored(rng.standard_normal((d, wide)) / wide ** 0.5)
    x = L.stored(rng.standard_normal((L.T, d)))
    xin = torch.empty(L.T, rows, dtype=L.tdt, device="cuda")
    B.ssm_gemm_nt(L.dev(x), L.dev(w_in), xin)                      # [q | k | v | z | b a]
    qkv_w = 256 + wide
    qkv, z = xin[:, :qkv_w], xin[:, qkv_w:qkv_w + wide]
    b, a = xin[:, qkv_w + wide:qkv_w + wide + 4], xin[:, qkv_w + wide + 4:]
    dd = L.desc(B)
    pool, o = L.dev(L.pool, False), torch.empty(L.T, wide, dtype=L.tdt, device="cuda")
    ws = B.workspace(B.delta_workspace_bytes(dd, L.T, L.n))
    B.ssm_delta_prefill(dd, L.gates(B, dd), qkv, a, b, B.SeqMeta(L.cu, L.slots, L.init, L.S), pool, o, ws)
    L.qkv = f64(qkv)
    L.proj = np.concatenate([f64(z), f64(b), f64(a)], 1)
    want, _, sizes = L.oracle()
    near(f64(o).reshape(want.shape), want, out_bound(want, sizes, act), "rule")
    w = (1 + 0.1 * rng.standard_normal(64)).astype(np.float32)
    before = f64(o).reshape(want.shape)
    B.ssm_gated_rmsnorm(o, B.GatedNorm(L.dev(w, False), z, 4, 64), o)      # in place
    y = od.head_norm(before, w.astype(np.float64), f64(z).reshape(want.shape), 1e-5)
    half = 2.0 ** -8 if act == "bf16" else 2.0 ** -24
    near(f64(o).reshape(want.shape), y, (half + 16 * 2.0 ** -24) * np.abs(y) + 1e-30, "head norm")
    part = torch.empty(L.T, d, dtype=L.tdt, device="cuda")
    B.ssm_gemm_nt(o, L.dev(w_out), part)
    res, normed = torch.from_numpy(x).cuda().float(), torch.empty(L.T, d, dtype=L.tdt, device="cuda")
    wp, wn = ((1 + 0.1 * rng.standard_normal(d)).astype(np.float32) for _ in range(2))
    B.ssm_block_rmsnorm(res, [part], res, L.dev(wn, False), 1e-5, normed, post_w=L.dev(wp, False), scale=0.5)
    r, nm = od.block_norm(x.astype(np.float64), [f64(part)], wn.astype(np.float64), 1e-5, post_w=wp.astype(np.float64), scale=0.5)
    near(f64(res), r, 24 * 2.0 ** -24 * (np.abs(r) + np.abs(r - x)) + 1e-30, "residual")
    near(f64(normed), nm, half * np.abs(nm) + 64 * 2.0 ** -24 * (np.abs(nm) + 1), "next norm")
    assert B.take_status(ws) == 0
