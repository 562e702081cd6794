"""The gated norm of heads and the norms between two blocks on the GPU against the float64 oracle."""
import numpy as np
import pytest

from delta_cases import f64, near
from oracle import delta as od

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _half(act):
    return 2.0 ** -8 if act == "bf16" else 2.0 ** -24


def _bound(y, act, steps=24):
    """One rounding of the value and `steps` float32 steps of products, exponentials and the mean in front of it. A sum
    of squares has no cancellation, and its relative error is halved by the root."""
    return (_half(act) + steps * 2.0 ** -24) * np.abs(y) + 1e-30


@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,dim", [(1, 1, 8), (3, 5, 16), (7, 2, 24), (257, 3, 48), (5, 16, 128), (2, 1, 504), (3, 2, 520),
                                            (2, 1, 2048), (1000, 12, 64), (4, 512, 8)])
@pytest.mark.parametrize("gate,first,per_head", [("silu", False, False), ("sigmoid", True, True), ("tanh", False, True),
                                                 ("identity", True, False), (None, False, False)])
def test_gated_norm(rows, heads, dim, gate, first, per_head, act):
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(rows + dim)
    n = heads * dim
    buf = torch.from_numpy(rng.standard_normal((rows, 2 * n + 16)).astype(np.float32)).to(DT[act]).cuda()
    x, z = buf[:, :n], buf[:, n + 8:2 * n + 8]                       # columns of one buffer
    w = (1 + 0.3 * rng.standard_normal(n if per_head else dim)).astype(np.float32)
    norm = B.GatedNorm(torch.from_numpy(w).cuda(), z if gate else None, heads, dim, eps=1e-4, gate=gate or "silu", gate_first=first)
    wide = torch.full((rows, n + 8), float("nan"), dtype=DT[act], device="cuda")
    B.ssm_gated_rmsnorm(x, norm, wide[:, :n])
    y = od.head_norm(f64(x).reshape(rows, heads, dim), w.astype(np.float64).reshape(-1, dim),
                     f64(z).reshape(rows, heads, dim) if gate else None, 1e-4, gate or "silu", first)
    # silu and sigmoid go through exp2(-z log2 e), whose argument is rounded: |z| 2^-24 more, and |z| stays below 6 here
    near(f64(wide[:, :n]).reshape(y.shape), y, _bound(y, act, 32), "out")
    assert torch.isnan(wide[:, n:]).all()
    kept = buf.clone()
    B.ssm_gated_rmsnorm(x, norm, x)                                  # in place
    assert torch.equal(x, wide[:, :n])
    kept[:, :n] = x
    assert torch.equal(buf, kept)


def test_gated_norm_of_zero_rows_and_far_gates():
    from paper_2602_21144_amd import binding as B
    x = torch.zeros(2, 64, device="cuda")
    x[1] = 1e15
    z = torch.tensor([-1e4, 1e4] * 32, device="cuda").expand(2, 64).contiguous()
    out = torch.empty_like(x)
    B.ssm_gated_rmsnorm(x, B.GatedNorm(torch.ones(64, device="cuda"), z, 1, 64), out)
    want = od.head_norm(np.array([[0.0] * 64, [1e15] * 64]), np.ones(64), np.array([[-1e4, 1e4] * 32] * 2) * np.array([[0, 1]] * 32).reshape(-1), 1e-5)
    near(f64(out), want, 32 * 2.0 ** -24 * np.abs(want) + 1e-30, "out")


BLOCKS = [(1, 8), (3, 24), (5, 768), (2, 1000), (4, 2048), (3, 2056), (2, 8192), (300, 320)]


@pytest.mark.parametrize("rows,d", BLOCKS)
@pytest.mark.parametrize("act", ["bf16", "f32"])
@pytest.mark.parametrize("n_parts,post,gate,fn,scale,inplace", [
    (1, True, None, "identity", 1.0, True), (2, False, "token", "sigmoid", 0.5, False), (8, True, "row", "tanh", -0.25, False),
    (0, True, None, "identity", 1.0, False), (3, False, None, "identity", 1.0, True), (1, True, "token", "silu", 2.0, True)])
def test_block_norm(rows, d, act, n_parts, post, gate, fn, scale, inplace):
    from paper_2602_21144_amd import binding as B
    rng = np.random.default_rng(rows + d + n_parts)
    mk = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DT[act]).cuda()  # noqa: E731
    base = mk(rows, d).float() if inplace or act == "f32" else mk(rows, d)
    parts = [mk(rows, d) for _ in range(n_parts)]
    wide = mk(rows if gate == "token" else 1, d + 8)
    g = wide[:, :d] if gate else None                                # strided rows
    post_w = torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).cuda() if post else None
    norm_w = torch.from_numpy((1 + 0.3 * rng.standard_normal(d)).astype(np.float32)).cuda()
    b64 = f64(base)
    res = base if inplace else torch.full((rows, d), float("nan"), device="cuda")
    normed = torch.full((rows, d), float("nan"), dtype=DT[act], device="cuda")
    B.ssm_block_rmsnorm(base, parts, res, norm_w, 1e-5, normed, post_w=post_w, post_eps=1e-3, gate=g, gate_fn=fn, scale=scale)
    p64 = [f64(p) for p in parts]
    r, nm = od.block_norm(b64, p64, f64(norm_w), 1e-5, post_w=f64(post_w) if post else None, post_eps=1e-3,
                          g=f64(g) if gate else None, fn=fn, scale=scale)
    # the sum of the parts is off by n steps of what is added up; norm, gate and scale multiply it
    size = sum([np.abs(p) for p in p64], np.zeros((rows, d)))
    y = np.abs(r - b64)
    total = np.abs(sum(p64, np.zeros((rows, d))))
    with np.errstate(invalid="ignore", divide="ignore"):
        factor = np.where(total > 0, y / total, 0.0)
    tol = 2.0 ** -24 * (np.abs(r) + 40 * y + n_parts * size * factor) + 1e-30
    near(f64(res), r, tol, "residual")
    inv = np.abs(nm) / np.maximum(np.abs(r), 1e-30)
    rel = np.sqrt((tol * tol).mean(-1, keepdims=True) / np.maximum((r * r).mean(-1, keepdims=True), 1e-30))
    near(f64(normed), nm, _bound(nm, act) + tol * inv + rel * np.abs(nm), "normed")


def test_block_norm_without_terms_is_the_residual_norm():
    """With no norm behind the block, no gate and a scale of one, the bits of ssm_residual_rmsnorm's residual."""
    from paper_2602_21144_amd import binding as B
    torch.manual_seed(1)
    base, parts = torch.randn(9, 2560, device="cuda"), [torch.randn(9, 2560, device="cuda").bfloat16() for _ in range(2)]
    w = torch.rand(2560, device="cuda")
    outs = []
    for f in (B.ssm_residual_rmsnorm, B.ssm_block_rmsnorm):
        res, normed = torch.empty_like(base), torch.empty(9, 2560, dtype=torch.bfloat16, device="cuda")
        f(base, parts, res, w, 1e-5, normed)
        outs.append((res, normed))
    assert torch.equal(outs[0][0], outs[1][0])
    assert (outs[0][1].float() - outs[1][1].float()).abs().max() <= 2.0 ** -7 * outs[0][1].float().abs().max()


def test_norms_captured_in_a_graph():
    from paper_2602_21144_amd import binding as B
    torch.manual_seed(2)
    x, z = (torch.randn(100, 256, device="cuda").bfloat16() for _ in range(2))
    out, res, normed = torch.empty_like(x), torch.zeros(100, 256, device="cuda"), torch.empty_like(x)
    w, wn = torch.rand(64, device="cuda"), torch.rand(256, device="cuda")
    s = torch.cuda.Stream()
    calls = [B.bind("ssm_gated_rmsnorm", x, B.GatedNorm(w, z, 4, 64), out, stream=s),
             B.bind("ssm_block_rmsnorm", res, [out], res, wn, 1e-5, normed, post_w=wn, gate=z, gate_fn="tanh", stream=s)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        for c in calls:
            c()
    ref = None
    for _ in range(3):
        res.zero_()
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, res, normed)]
        res.zero_()
        torch.cuda.synchronize()
        for c in calls:
            c()
        torch.cuda.synchronize()
        ref = [out, res, normed]
        assert all(torch.equal(p, q) for p, q in zip(got, ref))
