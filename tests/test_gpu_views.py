"""Rows as they lie: views that outlive the program's own reference to their cache, and rows of a view appended."""
import gc
import weakref

import numpy as np
import pytest
import torch

import paper_2605_12471_amd as kv
import qcache_ref as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hkv,n,at", [(1, 1, 3), (2, 1, 5), (1, 7, 2)])
def test_rows_of_odd_strides_that_mean_nothing(hkv, n, at):
    """One row, or one KV head, out of a tensor whose other stride is no multiple of 8."""
    k = torch.randn(n, hkv, 64).bfloat16()
    memory = torch.zeros(n * hkv * 64 + 8, dtype=torch.bfloat16, device="cuda")
    view = memory.as_strided((n, hkv, 64), (hkv * 64 if n > 1 else 8 * at + 1, 64 if hkv > 1 else at, 1))
    view.copy_(k)
    cache = kv.KvFoldQuantCache(1, 2, hkv, 64, 4, 20)
    cache.append(0, view, k.cuda())
    got = [torch.empty((n, hkv, 64), device="cuda") for _ in range(2)]
    cache.read(0, 0, *got)
    for x in got:
        assert np.array_equal(x.cpu().numpy(), R.held(k.float().numpy()).astype(np.float32))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_view_keeps_its_cache(dtype):
    cache = kv.KvFoldCache(1, 2, 2, 64, 8, 50, dtype)
    k, v = cache.view(0)
    known = weakref.ref(cache)
    del cache
    gc.collect()
    assert known() is not None          # (nothing is read before this is known)
    k.fill_(2.0)
    part = k[1, 3:5]
    del k, v
    gc.collect()
    assert known() is not None and (part == 2).all()
    gc.disable()
    try:
        del part
        assert known() is None          # (at once, not when rubbish is next collected)
    finally:
        gc.enable()
