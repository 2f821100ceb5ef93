"""The 8-bit cache's calls, weigh and evict through the Python binding: the native form and the plain Python one give the same results and the same errors."""
import pytest
import torch

import paper_2605_12471_amd as kv
from paper_2605_12471_amd import binding
from paper_2605_12471_amd import inputs as I

pytestmark = pytest.mark.gpu
HQ, HKV, D, N, PREV = 8, 2, 64, 12, 100


def both(make):
    """What make(cache) gives on a cache with the native calls and on one without."""
    got = []
    for native in (True, False):
        quant, cache = kv.KvFoldQuantCache(1, HQ, HKV, D, N, 200), kv.KvFoldCache(1, HQ, HKV, D, N, 200)
        if not native:
            quant._bound = cache._bound_weights = None
        else:
            assert binding._native_step() is not None
        g = torch.Generator().manual_seed(5)
        x = {name: torch.randn((n, h, D), generator=g).bfloat16().cuda() for name, n, h in (("q", N, HQ), ("k", N, HKV), ("v", N, HKV), ("pk", PREV, HKV), ("pv", PREV, HKV))}
        x["w"] = torch.rand((HKV, 200), generator=g).cuda()
        quant.append(0, x["pk"], x["pv"])
        for view, name in zip(cache.view(0), ("pk", "pv")):
            view[:, :PREV].copy_(x[name].transpose(0, 1))
        cache.set_length(0, PREV)
        try:
            r = make(quant, cache, x)
            torch.cuda.synchronize()
            got.append([t.float().cpu() if isinstance(t, torch.Tensor) else t for t in r])
        except (kv.KvFoldError, ValueError) as e:
            got.append([type(e), getattr(e, "status", None)])
    for a, b in zip(*got):
        assert torch.equal(a, b) if isinstance(a, torch.Tensor) else a == b
    return got[0]


@pytest.mark.parametrize("rope", [False, True])
@pytest.mark.parametrize("stream", [False, True])
def test_step_and_read(rope, stream):
    def make(quant, cache, x):
        out, lse = torch.empty_like(x["q"]), torch.empty((HQ, N), device="cuda")
        angles = tuple(t.cuda() for t in I.rope_tables(D, PREV, N)) if rope else None
        torch.cuda.synchronize()
        s = torch.cuda.Stream().cuda_stream if stream else None
        assert quant.step(0, x["q"], x["k"], x["v"], out, lse=lse, rope=angles, stream=s) is out
        torch.cuda.synchronize()
        k, v = (torch.empty((20, HKV, D), device="cuda") for _ in range(2))
        quant.read(0, 60, k, v)
        only = torch.empty((3, HKV, D), device="cuda")
        quant.read(0, 109, None, only)
        return out, lse, k, v, only, quant.length(0)
    both(make)


def test_weigh_and_evict():
    def make(quant, cache, x):
        lse = torch.full((HQ, N), 3.0, device="cuda")
        w = cache.weigh(0, x["q"], lse, x["w"].clone())
        w2 = cache.weigh(0, x["q"], lse, x["w"].clone(), add=False, rope=tuple(t.cuda() for t in I.rope_tables(D, 88, N)))
        to = kv.KvFoldCache(2, HQ, HKV, D, N, 60)
        to_w = torch.empty((HKV, 60), device="cuda")
        kept = cache.evict(0, w, 50, 2, 10, to=to, to_layer=1, to_weights=to_w)
        here = cache.evict(0, w, 70, 0, 0, to_weights=w, kept=torch.empty((HKV, 70), dtype=torch.int32, device="cuda"),
                           workspace=torch.empty(cache.evict_workspace_bytes(70), dtype=torch.uint8, device="cuda"))
        return [w, w2, to_w, kept, here, *(t[:, :50].clone() for t in to.view(1)), *(t[:, :70].clone() for t in cache.view(0)), cache.length(0), to.length(1)]
    both(make)


@pytest.mark.parametrize("call", [
    lambda quant, cache, x: quant.step(0, x["q"], x["k"], x["v"], torch.empty_like(x["q"]), pos_offset=3),
    lambda quant, cache, x: quant.step(1, x["q"], x["k"], x["v"], torch.empty_like(x["q"]), pos_offset=3),
    lambda quant, cache, x: quant.step(0, x["q"].float(), x["k"], x["v"], torch.empty_like(x["q"])),
    lambda quant, cache, x: quant.step(0, x["q"], x["k"][:3], x["v"], torch.empty_like(x["q"])),
    lambda quant, cache, x: quant.step(0, x["q"][:0], x["k"][:0], x["v"][:0], x["q"][:0]),
    lambda quant, cache, x: quant.step(0, x["q"].cpu(), x["k"], x["v"], torch.empty_like(x["q"])),
    lambda quant, cache, x: quant.read(0, 90, torch.empty((11, HKV, D), device="cuda"), None),
    lambda quant, cache, x: quant.read(0, -1, torch.empty((2, HKV, D), device="cuda"), None),
    lambda quant, cache, x: quant.read(0, 0, torch.empty((2, HKV, D), device="cuda"), torch.empty((3, HKV, D), device="cuda")),
    lambda quant, cache, x: cache.weigh(0, x["q"], torch.zeros((HQ, N - 1), device="cuda"), x["w"]),
    lambda quant, cache, x: cache.weigh(3, x["q"], torch.zeros((HQ, N), device="cuda"), x["w"]),
    lambda quant, cache, x: cache.weigh(0, x["q"], torch.zeros((HQ, N), device="cuda"), x["w"][:, :100]),
    lambda quant, cache, x: cache.evict(0, x["w"], 101),
    lambda quant, cache, x: cache.evict(0, x["w"], 0),
    lambda quant, cache, x: cache.evict(0, x["w"], -5),
    lambda quant, cache, x: cache.evict(0, x["w"], 10, 11, 0),
    lambda quant, cache, x: cache.evict(0, x["w"], 10, kept=torch.empty((HKV, 9), dtype=torch.int32, device="cuda")),
    lambda quant, cache, x: cache.evict(0, x["w"], 10, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")),
])
def test_the_same_errors(call):
    got = both(lambda quant, cache, x: [call(quant, cache, x)])
    assert got[0] in (kv.KvFoldError, ValueError)


def test_a_closed_target_is_no_target():
    cache, to = kv.KvFoldCache(1, HQ, HKV, D, N, 100), kv.KvFoldCache(1, HQ, HKV, D, N, 100)
    cache.set_length(0, 50)
    to.close()
    with pytest.raises(ValueError):
        cache.evict(0, torch.zeros((HKV, 100), device="cuda"), 10, to=to)
    assert cache.length(0) == 50
