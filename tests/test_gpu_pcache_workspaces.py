"""A batch's workspace is for so many sequences and KV heads: a step with others is refused, in both forms of the binding."""
import pytest
import torch

import paper_2605_12471_amd as kv
from test_gpu_pcache import Fold

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("prev,new", [([9000, 40], [1, 1]), ([20, 3], [70, 40])])
def test_batches_of_other_caches_and_of_other_numbers_of_sequences(prev, new, native):
    f = Fold(8, 2, 128, 16, prev, new)
    f.step()
    if not native:
        f.cache._bound = None
    assert (f.cache._bound is not None) == native
    q, k, v = f.dev
    for hq, hkv, taken in ((8, 8, False), (2, 2, True), (4, 1, False)):
        with kv.KvFoldPagedCache(1, hq, hkv, 128, 16, f.n_pages) as other:
            if not native:
                other._bound = None
            shapes = [torch.zeros((f.rows, heads, 128), dtype=torch.bfloat16, device="cuda") for heads in (hq, hkv, hkv, hq)]
            if taken:  # (as many KV heads: one workspace serves both)
                other.step(0, f.batch, *shapes)
            else:
                with pytest.raises(ValueError):
                    other.step(0, f.batch, *shapes)
    b = f.batch
    kept = b.tables, b.lens, b.cu_new
    b.tables, b.lens, b.cu_new = b.tables[:1].clone(), b.lens[:1].clone(), b.cu_new[:2].clone()
    with pytest.raises(ValueError):
        f.step()
    b.tables, b.lens, b.cu_new = kept
    f.cache.view(0)[0].copy_(f.k_pages)
    f.cache.view(0)[1].copy_(f.v_pages)
    f.step().check().check_pages()
