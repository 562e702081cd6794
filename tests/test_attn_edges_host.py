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
