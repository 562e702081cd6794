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
