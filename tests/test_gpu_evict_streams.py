"""Eviction on a stream that is handed in, with memory that the call takes by itself."""
import pytest
import torch

import paper_2605_12471_amd as kv

pytestmark = pytest.mark.gpu
HQ, HKV, D, ROWS = 8, 2, 64, 3000


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("in_place", [False, True])
def test_memory_taken_beside_a_late_eviction_is_other_memory(native, in_place):
    """The stream is busy with something else first, and the current stream goes on with tensors of the sizes that the eviction took."""
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((HKV, ROWS, D), generator=g).bfloat16().cuda() for _ in range(2))
    weights = torch.rand((HKV, ROWS), generator=g).cuda()
    order = torch.sort(weights, dim=-1, descending=True, stable=True).indices[:, :1000]
    want = torch.sort(order, dim=-1).values
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    for _ in range(3):
        cache, to = kv.KvFoldCache(1, HQ, HKV, D, 16, ROWS), None if in_place else kv.KvFoldCache(1, HQ, HKV, D, 16, 1000)
        if not native:
            cache._bound_weights = None
        for rows, x in zip(cache.view(0), (k, v)):
            rows.copy_(x)
        cache.set_length(0, ROWS)
        need = cache.evict_workspace_bytes(1000)
        # what the current stream has let go is there to be given out again
        free = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in (need, HKV * 1000 * 4) for _ in range(4)]
        del free
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(8):
                busy = busy @ busy * 1e-2
        kept = cache.evict(0, weights, 1000, to=to, stream=side.cuda_stream)
        others = [torch.full((n,), 0xff, dtype=torch.uint8, device="cuda") for n in (need, HKV * 1000 * 4) for _ in range(8)]
        torch.cuda.current_stream().synchronize()
        side.synchronize()
        assert torch.equal(kept.long(), want)
        index = want[:, :, None].expand(-1, -1, D)
        for rows, x in zip((cache if in_place else to).view(0), (k, v)):
            assert torch.equal(rows[:, :1000], torch.gather(x, 1, index))
        assert all((t == 0xff).all() for t in others)
