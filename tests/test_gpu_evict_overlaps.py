"""What an eviction writes may not lie in any layer's rows, of the cache or of the one that it moves them to."""
import pytest
import torch

import paper_2605_12471_amd as kv

pytestmark = pytest.mark.gpu
HKV, D, ROWS, KEEP = 2, 64, 200, 50


@pytest.mark.parametrize("what", ["kept", "workspace", "to_weights"])
@pytest.mark.parametrize("where", ["another layer of the cache", "another layer of the target", "the last bytes of the cache"])
def test_results_in_other_layers_rows(what, where):
    cache, to = kv.KvFoldCache(3, 4, HKV, D, 8, ROWS), kv.KvFoldCache(2, 4, HKV, D, 8, ROWS)
    for c in (cache, to):
        for layer in range(c.cfg.n_layers):
            for rows in c.view(layer):
                rows.fill_(3.0)
    cache.set_length(-1, ROWS)
    weights = torch.rand((HKV, ROWS), device="cuda")
    need = cache.evict_workspace_bytes(KEEP)
    kept, space, to_weights = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (HKV * KEEP * 4, need, HKV * ROWS * 4))
    size = {"kept": kept, "workspace": space, "to_weights": to_weights}[what].numel()
    v_end = lambda c, layer: c.view(layer)[1].data_ptr() + HKV * ROWS * D * 2
    at = {"another layer of the cache": cache.view(1)[0].data_ptr() + 256, "another layer of the target": to.view(0)[1].data_ptr(),
          "the last bytes of the cache": v_end(cache, 2) - 256}[where]
    if where == "the last bytes of the cache":
        at = v_end(cache, 2) - size // 256 * 256 - 256
    place = {"kept": kept.data_ptr(), "workspace": space.data_ptr(), "to_weights": to_weights.data_ptr(), what: at}
    rc = kv.kvfold_cache_evict(cache.handle, 0, weights.data_ptr(), KEEP, 2, 3, to.handle, 1, place["to_weights"], place["kept"], place["workspace"], need)
    torch.cuda.synchronize()
    assert rc == -1 and to.length(1) == 0
    for c in (cache, to):
        for layer in range(c.cfg.n_layers):
            assert all((rows == 3.0).all() for rows in c.view(layer))
    assert kv.kvfold_cache_evict(cache.handle, 0, weights.data_ptr(), KEEP, 2, 3, to.handle, 1, to_weights.data_ptr(), kept.data_ptr(), space.data_ptr(), need) == 0
    torch.cuda.synchronize()
