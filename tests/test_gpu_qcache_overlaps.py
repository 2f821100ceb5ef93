"""Rows read back onto the cache's own storage or onto one another, and rows to append that lie in it, are refused."""
import pytest
import torch

import paper_2605_12471_amd as kv
from paper_2605_12471_amd import binding

pytestmark = pytest.mark.gpu
HKV, D = 2, 64


def test_refused_before_anything_is_enqueued():
    cfg = binding.make_config(2, 4, HKV, D, 64, 300, kv.KVFOLD_BF16)
    need = kv.kvfold_qcache_bytes_required(cfg)
    buf = torch.zeros(need + 512, dtype=torch.uint8, device="cuda")
    base = (buf.data_ptr() + 255) // 256 * 256
    cfg.kv_buffer, cfg.kv_buffer_bytes = base, need
    rc, h = kv.kvfold_qcache_create(cfg)
    assert rc == 0
    rows = torch.randn(200, HKV, D, device="cuda").bfloat16()
    assert kv.kvfold_qcache_append(h, 0, rows.data_ptr(), rows.data_ptr(), HKV * D, D, 200, 0) == 0   # (the same rows for both are none of it)
    torch.cuda.synchronize()
    held = buf.clone()
    out = torch.zeros((2, 200, HKV, D), device="cuda")
    k, v, size = out[0].data_ptr(), out[1].data_ptr(), 200 * HKV * D * 4
    for a, b in ((base, v), (k, base + need - 256), (base + need - 16, None), (None, base), (k, k), (k, k + size - 16), (k + size - 16, k)):
        assert kv.kvfold_qcache_read(h, 0, 0, 200, a, b) == -1
    for a, b in ((base, rows.data_ptr()), (rows.data_ptr(), base + need - 256)):
        assert kv.kvfold_qcache_append(h, 1, a, b, HKV * D, D, 10, 0) == -1
    # rows [Hkv][capacity][d] whose last head is the one that lies there
    assert kv.kvfold_qcache_append(h, 1, base - 4096, rows.data_ptr(), D, 2048, 1, 0) == -1
    # a step's inputs
    q, kn, vn, o = (torch.ones((4, n, D), device="cuda", dtype=torch.bfloat16) for n in (4, HKV, HKV, 4))
    for name, at in (("q", base), ("k", base + need - 512), ("v", base + need // 256 // 2 * 256)):
        place = {"q": q.data_ptr(), "k": kn.data_ptr(), "v": vn.data_ptr(), name: at}
        assert kv.kvfold_qcache_step(h, 0, place["q"], place["k"], place["v"], 4, 200, None, None, o.data_ptr()) == -1
    torch.cuda.synchronize()
    assert (o == 1).all() and kv.kvfold_qcache_length(h, 0) == 200
    assert torch.equal(buf, held) and kv.kvfold_qcache_length(h, 1) == 0 and not out.any()
    assert kv.kvfold_qcache_read(h, 0, 0, 200, k, v) == 0 and kv.kvfold_qcache_read(h, 0, 0, 0, base, base) == 0
    torch.cuda.synchronize()
    assert kv.kvfold_qcache_destroy(h) == 0
