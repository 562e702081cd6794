"""Prompts of the gated delta rule where values, states, write strengths and decays of one call lie far apart: the state
keeps float32's precision whatever a chunk holds beside the tokens that make it, and an output is rounded once."""
import numpy as np
import pytest

from delta_cases import Layer, f64, near, state_bound
from test_gpu_delta import HEADS, LENS, _prefill

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# a workgroup with waves of their own for the outputs, and one without; more sequences than run at once by twos
SHAPES = [("bf16", (1, 2, 64, 64)), ("bf16", (2, 2, 128, 128)), ("bf16", (1, 1, 144, 32)), ("bf16", (1, 1, 256, 48)),
          ("f32", (1, 2, 64, 64)), ("f32", (1, 1, 128, 64)), ("f32", (1, 1, 256, 48))]


def once_bound(want, sizes, act):
    """What out_bound gives float32 outputs, for both types: sums, states and their operands have float32's precision
    (128 times 2^-24 of what is summed, see there), and one rounding of the value to its type stands behind them. What
    out_bound leaves bf16 beyond that, for operands of 11 bits, none of them needs."""
    return (2.0 ** -8 if act == "bf16" else 2.0 ** -24) * np.abs(want) + 128 * 2.0 ** -24 * sizes + 1e-30


def _layer(act, heads, lens, log_alpha=-0.5, seed=50, **kw):
    """Every token's decay is e^log_alpha, as the activation type holds it."""
    L = Layer(torch, heads, lens, act, seed=seed, **kw)
    L.A_log[:], L.dt_bias[:] = 0.0, 0.0
    _, b, a = L.columns(L.proj)
    a[:] = L.stored(np.full(a.shape, np.log(np.expm1(-log_alpha))))
    return L, b, a


def _hold(L, what=""):
    out, pool, status, _ = _prefill(L)
    assert status == 0
    o, want, sizes = L.oracle()
    near(f64(pool)[L.slots], want[L.slots], state_bound(want[L.slots], L.act), f"{what} state")
    near(f64(out).reshape(o.shape), o, once_bound(o, sizes, L.act), f"{what} out")


@pytest.mark.parametrize("act,heads", SHAPES, ids=str)
@pytest.mark.parametrize("log_alpha,closed", [(-0.5, -6.0), (-1.6, -8.0), (-1.6, -12.0)])
def test_write_gates_that_close(log_alpha, closed, act, heads):
    """Write strengths of e^-6 to e^-12 for the last tokens of a chunk, beside ordinary ones that the decay leaves little of."""
    L, b, _ = _layer(act, heads, [64, 116], log_alpha, init=[0, 1])
    for lo in (52, 64 + 52, 128 + 40):
        b[lo:lo + 12] = closed
    _hold(L)


@pytest.mark.parametrize("act,heads", SHAPES, ids=str)
@pytest.mark.parametrize("closed", [-8.0, -16.0, -28.0])
def test_write_gates_that_are_closed_behind_a_reset(closed, act, heads):
    L, b, a = _layer(act, heads, [64, 130])
    for at in (20, 64 + 20, 64 + 84):
        a[at] = 10000.0
    b[20:64] = b[84:128] = b[148:] = closed
    _hold(L)


@pytest.mark.parametrize("act,heads", SHAPES, ids=str)
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20, 2.0 ** 40])
def test_large_values_in_front_of_a_reset(size, act, heads):
    L, _, a = _layer(act, heads, [64, 130])
    hk, hv, dk, dv = heads
    L.qkv[[3, 70], 2 * hk * dk:] = L.stored(L.qkv[[3, 70], 2 * hk * dk:] * size)
    a[[9, 64 + 20]] = 10000.0
    _hold(L)


@pytest.mark.parametrize("act,heads", SHAPES, ids=str)
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 20, 2.0 ** 40])
def test_a_large_state_in_front_of_a_reset(size, act, heads):
    L, _, a = _layer(act, heads, [64, 130], init=[1, 1])
    L.pool *= np.float32(size)
    a[[1, 64 + 33]] = 10000.0
    _hold(L)


@pytest.mark.parametrize("act,heads", SHAPES, ids=str)
def test_short_keys_beside_long_ones(act, heads):
    """Keys of the program's own lengths: those behind a reset are 2^-30 as long as those in front of it."""
    L, _, a = _layer(act, heads, [64, 100], qk_norm=False)
    hk, hv, dk, dv = heads
    k = L.qkv[:, hk * dk:2 * hk * dk]
    for lo, hi in ((20, 64), (64 + 11, 128), (64 + 70, 164)):
        k[lo:hi] *= np.float32(2.0 ** -30)
        a[lo] = 10000.0
    _hold(L)


@pytest.mark.parametrize("act,heads", SHAPES, ids=str)
def test_keys_whose_squares_vanish(act, heads):
    """Keys of 2^-76, whose squares are below float32, and no values: what is taken off the state is small, not
    infinite."""
    L, _, _ = _layer(act, heads, [70], -0.01, init=[1], qk_norm=False)
    hk, hv, dk, dv = heads
    L.qkv[:, hk * dk:2 * hk * dk] *= np.float32(2.0 ** -76)
    L.qkv[:, 2 * hk * dk:] = 0.0
    _hold(L)


@pytest.mark.parametrize("act,heads", SHAPES, ids=str)
@pytest.mark.parametrize("size", [2.0 ** 105, 2.0 ** -60])
def test_values_and_states_at_the_ends_of_their_range(size, act, heads):
    L, _, _ = _layer(act, heads, [64, 100], -0.05, init=[0, 1])
    hk, hv, dk, dv = heads
    L.qkv[:, 2 * hk * dk:] = L.stored(L.qkv[:, 2 * hk * dk:] * size)
    L.pool *= np.float32(size)
    _hold(L)


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_an_output_is_rounded_once(heads, lens, act):
    L = Layer(torch, heads, lens, act, seed=60 + len(lens) + heads[2])
    _hold(L)


@pytest.mark.parametrize("act,heads,lens", [("bf16", (16, 32, 128, 128), [70, 1, 65, 3, 128, 64, 90, 2, 70, 64]),
                                            ("f32", (64, 64, 32, 48), [20, 3, 65, 70, 1, 2]), ("bf16", (4, 12, 192, 192), [64, 100, 1, 70] * 6)],
                         ids=str)
def test_outputs_of_many_heads_are_rounded_once(act, heads, lens):
    """By workgroups of four waves of columns."""
    L = Layer(torch, heads, lens, act, seed=61, init=[i % 2 for i in range(len(lens))])
    _hold(L)


@pytest.mark.parametrize("act,heads", [("bf16", (16, 32, 64, 64)), ("f32", (16, 32, 64, 64)), ("f32", (16, 32, 96, 64)), ("bf16", (16, 32, 144, 64))],
                         ids=str)
def test_resets_in_many_heads(act, heads):
    """The closed gates and the large values above, by workgroups of four waves of columns."""
    L, b, a = _layer(act, heads, [64, 130, 5, 70, 66, 64, 1, 3, 64, 20])
    hk, hv, dk, dv = heads
    for lo in L.cu[:-1]:
        hi = min(lo + 64, L.T)
        L.qkv[lo, 2 * hk * dk:] = L.stored(L.qkv[lo, 2 * hk * dk:] * 2.0 ** 20)
        a[min(lo + 2, hi - 1)] = 10000.0
        b[min(lo + 2, hi - 1):hi] = -10.0
    _hold(L)



@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["q", "k", "a", "b", "state"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_value_that_is_not_finite_stays_in_its_sequence(value, what, act):
    """In a sequence between two others: those and what lies more than 63 rows in front keep their values; for the gates
    and a state so do the other value heads of the same keys."""
    L, b, a = _layer(act, (1, 2, 64, 64), [90, 200, 64], init=[1, 1, 1])
    o, want, sizes = L.oracle()
    at, pool = 90 + 150, L.pool.copy()
    if what == "q":
        L.qkv[at, 7] = value
    elif what == "k":
        L.qkv[at, 64 + 7] = value
    elif what == "state":
        L.pool[L.slots[1], 1, 5, 9] = value
        at = 90
    else:
        # an infinite decay forgets everything and an infinite write strength is 1: both are ordinary
        (a if what == "a" else b)[at, 1] = float("nan")
    out, got_pool, status, _ = _prefill(L)
    assert status == 0
    got, tol = f64(out).reshape(o.shape), once_bound(o, sizes, act)
    rows = np.r_[0:max(at - 63, 90), 290:354]
    near(got[rows], o[rows], tol[rows], "rows of others")
    if what in ("a", "b", "state"):
        near(got[:, 0], o[:, 0], tol[:, 0], "the other head")
        assert not np.isfinite(got[at, 1]).all()
    else:
        assert not np.isfinite(got[at]).any()
    st, bound = f64(got_pool), state_bound(want, act)
    others = [L.slots[0], L.slots[2]]
    near(st[others], want[others], bound[others], "states of others")
    assert np.isfinite(st[L.slots[1]]).all() == (what == "q")
    spare = [s for s in range(L.S) if s not in L.slots]
    assert np.array_equal(st[spare], pool[spare].astype(np.float64))


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("n,overlap", [(3, False), (64, True), (300, True), (300, False)])
def test_nothing_is_written_behind_the_workspace(n, overlap, act):
    """A workspace of the exact size in front of a filled region. Where every second sequence names all rows of the call
    there are far more chunks than a call of that many rows has, laid out by the first launch (up to 256 sequences) or
    by one of its own."""
    from paper_2602_21144_amd import binding as B
    T = 640
    L = Layer(torch, (1, 2, 32, 16), [T] + [0] * (n - 1) if overlap else [T // n] * n, act, seed=13)
    dd = L.desc(B)
    meta = B.SeqMeta(L.cu, L.slots, L.init, L.S)
    if overlap:
        meta.cu.copy_(torch.tensor([0, T] * (n // 2) + [0], dtype=torch.int32))
    need = B.delta_workspace_bytes(dd, L.T, n)
    buf = torch.full((need + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
    ws = buf[:need]
    ws.zero_()
    proj, pool = L.dev(L.proj), L.dev(L.pool, False)
    _, b, a = L.columns(proj)
    out = torch.empty(L.T, L.wide, dtype=L.tdt, device="cuda")
    B.ssm_delta_prefill(dd, L.gates(B, dd), L.dev(L.qkv), a, b, meta, pool, out, ws)
    torch.cuda.synchronize()
    assert (buf[need:] == 0xA5).all()
    assert bool(B.take_status(ws) & B.SSM_STATUS_BAD_SEQLENS) == overlap
    others = [s for s in range(L.S) if s not in L.slots]
    assert np.array_equal(f64(pool)[others], L.pool[others].astype(np.float64))
