"""Rows whose log-sum-exp is -inf count for nothing, whatever their queries are."""
import math

import pytest
import torch

import paper_2605_12471_amd as kv
from test_gpu_evict import TYPE, draw, filled

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,d,n,rows", [
    ("bf16", 8, 2, 128, 3, 500), ("bf16", 8, 8, 64, 16, 77), ("bf16", 8, 2, 64, 40, 900), ("bf16", 28, 4, 128, 33, 700), ("bf16", 8, 2, 128, 100, 900),
    ("bf16", 32, 2, 64, 64, 64), ("f32", 4, 1, 64, 5, 300), ("f32", 4, 1, 128, 20, 300), ("f32", 4, 1, 64, 60, 300), ("f32", 6, 2, 128, 43, 43)])
@pytest.mark.parametrize("rope", [False, True])
def test_rows_that_do_not_count(dtype, hq, hkv, d, n, rows, rope):
    """Padding whose queries were never written: NaN and infinities there leave the bits of zeros there.  All rows, the last ones, and some between."""
    cache, _, _ = filled(hq, hkv, d, rows, dtype, seed=4)
    q, lse = draw((n, hq, d), 1, dtype), torch.randn((hq, n), generator=torch.Generator().manual_seed(2)) + 5
    angles = tuple(torch.rand((n, d // 2), generator=torch.Generator().manual_seed(s)).cuda() for s in (6, 7)) if rope else None
    for off in (torch.ones(n, dtype=torch.bool), torch.arange(n) >= n - 2, torch.arange(n) % 3 == 1):
        x, y = q.clone(), q.clone()
        x[off], y[off] = 0, torch.tensor([math.nan, math.inf, -math.inf, 1.0]).to(TYPE[dtype])[torch.arange(d) % 4]
        m = lse.clone()
        m[:, off] = -math.inf
        got = [cache.weigh(0, t.cuda(), m.cuda(), torch.zeros((hkv, rows), device="cuda"), add=False, rope=angles) for t in (x, y)]
        assert torch.isfinite(got[0]).all() and torch.isfinite(got[1]).all() and torch.equal(got[0], got[1])
        assert got[0].any() == (not off.all())
    # one head alone of a token
    m, y = lse.clone(), q.clone()
    m[hq - 1, n - 1], y[n - 1, hq - 1] = -math.inf, math.nan
    got = cache.weigh(0, y.cuda(), m.cuda(), torch.zeros((hkv, rows), device="cuda"), add=False, rope=angles)
    assert torch.isfinite(got).all() and got.any()
