"""The plain form that takes a chunk and head at a time against the one that goes row by row, and its values against the format's."""
import math

import numpy as np
import pytest
import torch

from paper_2601_18401_amd import binding as B
from tests import fp4_reference as fp4
from tests import paged_reference as ref
from tests import paged_whole_reference as whole


def i32(v):
    return torch.tensor(v, dtype=torch.int32)


@pytest.mark.parametrize("held", ["4 bits", "rows"])
@pytest.mark.parametrize("topk,S", [(0, 1000), (3, 10), (4, 7)])
def test_it_agrees_with_the_form_row_by_row(held, topk, S):
    g = torch.Generator().manual_seed(S)
    Hq, Hkv, D, ps, Ls, cu = 6, 2, 64, 9, [40, 7, 61], [0, 5, 8, 20]
    if held == "rows":
        K, V = (torch.randn((1, 20, Hkv, ps, D), generator=g) for _ in range(2))
    else:
        K, V = (torch.randint(0, 256, (1, 20, Hkv, B.PageCache.page_bytes(ps, D)), generator=g, dtype=torch.uint8) for _ in range(2))
        for x in (K, V):
            x[..., ps * (D // 2):] = 125 + x[..., ps * (D // 2):] % 3
    tables = torch.randperm(20, generator=g)[:18].int().view(3, 6).repeat(1, 2)
    tables[0, 2], tables[2, 4] = -1, 99
    kw = dict(page_size=ps, D=D, dtype=torch.float32) if held == "4 bits" else {}
    cache = B.PageCache(K, V, tables, i32(Ls), i32([0] * 20), **kw)
    plain = [fp4.values(x[0], ps, D) if held == "4 bits" else x[0] for x in (K, V)]
    assert all(torch.equal(whole.values(cache, name), x.double()) for name, x in zip("KV", plain))
    Q = torch.randn((Hq, 20, D), generator=g)
    idx = torch.stack([torch.randperm(9, generator=g)[:topk] for _ in range(Hq * 20)]).view(Hq, 20, topk).int() if topk else None
    if topk:
        idx[torch.rand(idx.shape, generator=g) < 0.3] = -1
    scores = torch.randn((Hq, 20, topk), generator=g) if topk else None
    for sc in [None] + [scores] * (topk > 0):
        O, A, LSE = whole.attention(cache, [0, 1, 2], cu, Q, idx, sc, S, L=50)
        wO, wL, wA = ref.attention(*plain, tables, cache.lens, [0, 1, 2], cu, Q, idx, sc, S, 1 / math.sqrt(D), 50)
        assert np.allclose(O, wO, rtol=1e-12, atol=1e-12) and np.allclose(A, wA, rtol=1e-12, atol=1e-12)
        assert sc is not None or np.allclose(LSE, wL, rtol=1e-12, atol=1e-12)


def test_a_block_that_is_nan_spoils_rows_that_attend_it():
    cache = B.PageCache.empty(1, 8, 1, 64, 1, 1, dtype=torch.float32, device="cpu", fp4=True)
    cache.tables[0, 0], cache.lens[0] = 0, 8
    for x in (cache.K, cache.V):
        x[..., 256:] = 126
    cache.V[0, 0, 0, 256 + 2 * 5 + 1] = 255      # token 5, channels 32 on
    O, _, LSE = whole.attention(cache, [0], [0, 8], torch.randn((1, 8, 64)), None, None, 100)
    assert torch.isfinite(LSE).all() and torch.equal(torch.isnan(O[0]), torch.outer(torch.arange(8) >= 5, torch.arange(64) >= 32))
    cache.K[0, 0, 0, 256 + 2 * 3] = 255          # token 3's key
    O, _, LSE = whole.attention(cache, [0], [0, 8], torch.randn((1, 8, 64)), None, None, 100)
    assert torch.isnan(O[0, 3:]).all() and torch.isnan(LSE[0, 3:]).all() and torch.isfinite(O[0, :3]).all()
