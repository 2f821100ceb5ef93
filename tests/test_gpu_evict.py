"""Attention weights by key, and eviction by them, on the GPU against their definitions."""
import math

import numpy as np
import pytest
import torch

import paper_2605_12471_amd as kv
from paper_2605_12471_amd import inputs as I

pytestmark = pytest.mark.gpu
TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def draw(shape, seed, dtype="bf16"):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(TYPE[dtype])


def filled(hq, hkv, d, rows, dtype="bf16", seed=0, capacity=None, chunk=None, layers=1):
    """A cache whose layers hold `rows` rows each; K, V [layers][Hkv][rows][d] on the host."""
    capacity = capacity or rows
    cache = kv.KvFoldCache(layers, hq, hkv, d, min(chunk or rows, capacity), capacity, dtype)
    k, v = draw((layers, hkv, rows, d), seed, dtype), draw((layers, hkv, rows, d), seed + 1, dtype)
    for layer in range(layers):
        for view, x in zip(cache.view(layer), (k, v)):
            view[:, :rows].copy_(x[layer])
    cache.set_length(-1, rows)
    return cache, k, v


def reference_weights(q, k, lse, d, group):
    """[Hkv][L] in 64 bits and what a kernel may be off by: every logit by (d + 2) 2^-24 of the sum of its products' magnitudes, the exponent by the
    roundings of the scale, of the log-sum-exp and of their difference, the exponential by 2^-22, the sum in fp32 by 2^-24 a row; a weight
    below fp32's smallest normal number may be lost."""
    n, hq, _ = q.shape
    hkv, length, _ = k.shape
    w, tol = np.zeros((hkv, length)), np.full((hkv, length), n * group * 2.0 ** -125)
    seen = np.arange(length)[None, :] <= length - n + np.arange(n)[:, None]
    for h in range(hq):
        kk, qq = k[h // group].double().numpy(), q[:, h].double().numpy()
        s, a = qq @ kk.T / math.sqrt(d), np.abs(qq) @ np.abs(kk).T / math.sqrt(d)
        m = lse[h].double().numpy()[:, None]
        p = np.where(seen & (m > -np.inf), np.exp(np.where(seen, s, 0) - np.where(m > -np.inf, m, 0)), 0)
        w[h // group] += p.sum(0)
        tol[h // group] += (p * ((d + 2) * 2.0 ** -24 * a + 2.0 ** -22 * (2 + np.abs(np.where(m > -np.inf, m, 0)) + a) + n * group * 2.0 ** -24)).sum(0)
    return w, tol


def log_sum_exp(q, k, d, group):
    n, hq, _ = q.shape
    length = k.shape[1]
    seen = torch.arange(length)[None, :] <= length - n + torch.arange(n)[:, None]
    return torch.stack([torch.logsumexp(torch.where(seen, q[:, h].double() @ k[h // group].double().T / math.sqrt(d), -math.inf), -1) for h in range(hq)]).float()


def check_weights(cache, q, k, lse, hq, hkv, d, rope=None, q_given=None):
    length, capacity = k.shape[1], cache.cfg.capacity_tokens
    weights = torch.full((hkv, capacity), 7.0, device="cuda")
    given = (q if q_given is None else q_given).cuda()
    assert cache.weigh(0, given, lse.cuda(), weights, add=False, rope=rope) is weights
    want, tol = reference_weights(q, k, lse, d, hq // hkv)
    got = weights.cpu().double().numpy()
    assert (got[:, length:] == 7).all()
    bad = np.argwhere(~(np.abs(got[:, :length] - want) <= tol))
    assert not len(bad), [(tuple(i), got[tuple(i)], want[tuple(i)], tol[tuple(i)]) for i in bad[:5]] + [len(bad)]
    first = weights.clone()
    cache.weigh(0, given, lse.cuda(), weights, rope=rope)
    assert torch.equal(weights[:, :length], first[:, :length] + first[:, :length]) and (weights[:, length:] == 7).all()
    return first


SHAPES = [(4, 1, 64), (8, 2, 128), (7, 1, 128), (3, 3, 64), (40, 2, 64), (6, 6, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("length,n", [(1, 1), (2, 2), (31, 1), (65, 3), (64, 64), (200, 5), (300, 150), (513, 40)])
def test_weights(dtype, hq, hkv, d, length, n):
    cache, k, _ = filled(hq, hkv, d, length, dtype, seed=length, capacity=length + 3, chunk=max(n, 2))
    q = draw((n, hq, d), length + 5, dtype)
    lse = log_sum_exp(q, k[0], d, hq // hkv)
    w = check_weights(cache, q, k[0], lse, hq, hkv, d)
    total = w[:, :length].double().sum(1).cpu()
    assert (total / (n * hq // hkv) - 1).abs().max() < 1e-5  # every row gives 1 (a rounding of the log-sum-exp, 2^-24 of at most 10, each)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("length,n", [(9001, 1), (5000, 3), (3000, 300)])
def test_weights_at_sizes_of_a_model(dtype, length, n):
    cache, k, _ = filled(28, 4, 128, length, dtype, seed=length, chunk=n)
    q = draw((n, 28, 128), length, dtype)
    check_weights(cache, q, k[0], log_sum_exp(q, k[0], 128, 7), 28, 4, 128)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,n", [(64, 1), (64, 40), (128, 2), (128, 33)])
def test_weights_behind_a_step_with_the_rotary_embedding(dtype, d, n):
    """A step leaves its log-sum-exps; its unrotated queries are rotated again."""
    hq, hkv, prev = 8, 2, 100
    cache, _, _ = filled(hq, hkv, d, prev, dtype, capacity=prev + n)
    q, kn, vn = (draw((n, h, d), i, dtype) for i, h in ((1, hq), (2, hkv), (3, hkv)))
    rope = tuple(t.cuda() for t in I.rope_tables(d, prev, n))
    lse = torch.empty((hq, n), device="cuda")
    cache.step(0, q.cuda(), kn.cuda(), vn.cuda(), torch.empty_like(q, device="cuda"), lse=lse, rope=rope)
    half = d // 2
    x, c, s = q.double(), rope[0].cpu().double()[:, None], rope[1].cpu().double()[:, None]
    lo, up = x[..., :half], x[..., half:]
    turned = torch.cat(((lo * c - (up * s).float().double()).float(), (up * c + (lo * s).float().double()).float()), -1).to(TYPE[dtype])
    torch.cuda.synchronize()
    check_weights(cache, turned, cache.view(0)[0].cpu(), lse.cpu(), hq, hkv, d, rope=rope, q_given=q)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 60])
def test_rows_that_count_for_nothing_and_keys_that_are_not_finite(dtype, n):
    """A log-sum-exp of -inf; keys that are not finite change only what sees them; the queries' units are filled up with nothing."""
    hq, hkv, d, length = 8, 2, 64, 200
    cache, k, _ = filled(hq, hkv, d, length, dtype)
    q = draw((n, hq, d), 5, dtype)
    lse = log_sum_exp(q, k[0], d, 4)
    lse[1, 0] = lse[7, n - 1] = -math.inf
    check_weights(cache, q, k[0], lse, hq, hkv, d)
    last = cache.view(0)[0]
    last[0, length - 1] = math.nan
    last[1, length - 1] = math.inf
    w = torch.zeros((hkv, length), device="cuda")
    cache.weigh(0, q.cuda(), lse.cuda(), w)
    want, tol = reference_weights(q, k[0], lse, d, 4)
    assert (np.abs(w.cpu().double().numpy() - want) <= tol)[:, :length - 1].all()


def test_logits_far_apart():
    cfg = I.FoldConfig("t", 78, 1, 8, 2, 64, 300, 300, "bf16")
    for profile in ("step100", "spike", "deep_start"):
        q, k, v = I.steered_qkv(cfg, 0, 0, profile, n_tokens=300, token_base=0)
        cache = kv.KvFoldCache(1, 8, 2, 64, 300, 300)
        cache.step(0, q.cuda(), k.cuda(), v.cuda(), torch.empty_like(q, device="cuda"))
        torch.cuda.synchronize()
        check_weights(cache, q, k.transpose(0, 1).contiguous(), log_sum_exp(q, k.transpose(0, 1), 64, 4), 8, 2, 64)


def kept_rows(w, keep, sink, recent):
    """Indices [Hkv][keep] by the definition: NaN above all, then by size, equal ones by the lowest index."""
    hkv, length = w.shape
    out = []
    for g in range(hkv):
        between = range(sink, length - recent)
        best = sorted(between, key=lambda j: (0 if math.isnan(w[g, j]) else 1, 0.0 if math.isnan(w[g, j]) else -w[g, j], j))[:keep - sink - recent]
        out.append(list(range(sink)) + sorted(best) + list(range(length - recent, length)))
    return np.array(out, dtype=np.int32).reshape(hkv, keep)


def same_bits(a, b):
    """(Memory that nothing was written to holds anything, NaN among it.)"""
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def run_evict(cache, k, v, w, keep, sink, recent, capacity, where, layer=0):
    """Evicts into the layer itself, another cache or another layer, and checks everything that there is afterwards."""
    layers, hkv, length, d = k.shape
    dtype = "f32" if k.dtype == torch.float32 else "bf16"
    want = kept_rows(w.numpy(), keep, sink, recent)
    full = torch.full((hkv, cache.cfg.capacity_tokens), 3.0)
    full[:, :length] = w
    full = full.cuda()
    before = [view.clone() for view in cache.view(layer)]
    if where == "here":
        to, to_layer, to_weights, args = cache, layer, full, {}
    elif where == "layer":
        to, to_layer, to_weights, args = cache, 1 - layer, torch.full_like(full, 5.0), dict(to=cache, to_layer=1 - layer)
    else:
        to, to_layer = kv.KvFoldCache(2, cache.cfg.n_q_heads, hkv, d, 1, capacity, dtype), 1
        to_weights, args = torch.full((hkv, capacity), 5.0, device="cuda"), dict(to=to, to_layer=1)
    target_before = [view.clone() for view in to.view(to_layer)]
    got = cache.evict(layer, full, keep, sink, recent, to_weights=to_weights, **args)
    torch.cuda.synchronize()
    assert np.array_equal(got.cpu().numpy(), want)
    index = torch.from_numpy(want).long()[:, :, None].expand(-1, -1, d)
    for view, rows, old in zip(to.view(to_layer), (k[layer], v[layer]), target_before):
        assert torch.equal(view[:, :keep].cpu(), torch.gather(rows, 1, index))
        assert same_bits(view[:, keep:], old[:, keep:])
    assert torch.equal(to_weights[:, :keep].cpu().view(torch.int32), torch.gather(w, 1, torch.from_numpy(want).long()).view(torch.int32))
    assert (to_weights[:, keep:] == 0).all()
    assert to.length(to_layer) == keep
    if where != "here":
        assert cache.length(layer) == length
        assert all(same_bits(a, b) for a, b in zip(cache.view(layer), before))
        assert torch.equal(full[:, :length].cpu().view(torch.int32), w.view(torch.int32))


def some_weights(hkv, length, seed, kind):
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(3 * torch.randn((hkv, length), generator=g) - 5)
    if kind == "ties":
        w = torch.randint(0, 4, (hkv, length), generator=g).float()
    elif kind == "equal":
        w = torch.zeros((hkv, length))
    elif kind == "odd":
        w[torch.rand((hkv, length), generator=g) < 0.2] = 0.0
        w[torch.rand((hkv, length), generator=g) < 0.2] = -0.0
        w[torch.rand((hkv, length), generator=g) < 0.1] *= -1
        w[torch.rand((hkv, length), generator=g) < 0.05] = math.nan
        w[torch.rand((hkv, length), generator=g) < 0.05] = math.inf
        w[torch.rand((hkv, length), generator=g) < 0.05] = -math.inf
        w[torch.rand((hkv, length), generator=g) < 0.1] = 1e-42
    return w


SIZES = [(1, 1, 0, 0), (2, 1, 0, 0), (64, 64, 0, 0), (65, 64, 1, 2), (200, 10, 4, 6), (200, 10, 0, 0), (1000, 700, 4, 32), (1000, 999, 0, 0), (1030, 129, 128, 0),
         (1030, 129, 0, 129), (5000, 64, 0, 1), (5000, 4100, 16, 1020)]


@pytest.mark.parametrize("where", ["here", "layer", "cache"])
@pytest.mark.parametrize("hkv,d,dtype", [(2, 64, "bf16"), (3, 128, "bf16"), (1, 128, "f32"), (2, 64, "f32")])
@pytest.mark.parametrize("length,keep,sink,recent", SIZES)
def test_evict(where, hkv, d, dtype, length, keep, sink, recent):
    cache, k, v = filled(hkv, hkv, d, length, dtype, capacity=length + 7, layers=2)
    run_evict(cache, k, v, some_weights(hkv, length, length, "plain"), keep, sink, recent, keep + 5, where)


@pytest.mark.parametrize("where", ["here", "cache"])
@pytest.mark.parametrize("kind", ["ties", "equal", "odd"])
@pytest.mark.parametrize("length,keep,sink,recent", [(3, 2, 0, 0), (300, 100, 4, 10), (2100, 1500, 0, 0), (2100, 70, 0, 3)])
def test_weights_that_are_equal_or_odd(where, kind, length, keep, sink, recent):
    cache, k, v = filled(2, 2, 64, length, layers=2)
    run_evict(cache, k, v, some_weights(2, length, length, kind), keep, sink, recent, keep, where)


@pytest.mark.parametrize("where", ["here", "cache"])
@pytest.mark.parametrize("keep", [20000, 39999, 300])
def test_a_long_cache(where, keep):
    cache, k, v = filled(8, 8, 128, 40000, layers=1)
    run_evict(cache, k, v, some_weights(8, 40000, 1, "plain"), keep, 4, 256, keep + 100, where)


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "odd"])
@pytest.mark.parametrize("length,keep,sink,recent", [(4096, 4000, 0, 0), (4097, 1, 0, 0), (8192, 100, 4, 8), (8193, 8192, 0, 0), (8193, 70, 60, 10), (16384, 9000, 8200, 5),
                                                     (20000, 16000, 0, 9000), (25000, 25000, 0, 0), (25000, 8300, 0, 8300), (33000, 12000, 1, 1)])
def test_rows_looked_through_by_one_or_several(kind, length, keep, sink, recent):
    cache, k, v = filled(2, 2, 64, length)
    run_evict(cache, k, v, some_weights(2, length, length, kind), keep, sink, recent, keep, "here")


@pytest.mark.parametrize("first", [True, False])
def test_the_kept_rows_are_the_first_or_the_last(first):
    """Nothing moves, or everything does, as far as it can."""
    length, keep = 6000, 3500
    cache, k, v = filled(2, 2, 128, length)
    w = torch.arange(length, 0, -1).float().repeat(2, 1) if first else torch.arange(length).float().repeat(2, 1)
    run_evict(cache, k, v, w, keep, 0, 0, keep, "here")


def test_evict_captured_and_on_another_stream():
    hkv, d, length, keep = 2, 64, 1500, 900
    cache, k, v = filled(hkv, hkv, d, length)
    w = some_weights(hkv, length, 3, "plain").cuda()
    to = kv.KvFoldCache(1, hkv, hkv, d, 1, keep)
    kept, to_weights = torch.empty((hkv, keep), dtype=torch.int32, device="cuda"), torch.empty((hkv, keep), device="cuda")
    space = torch.full((cache.evict_workspace_bytes(keep),), 0xff, dtype=torch.uint8, device="cuda")
    call = lambda: cache.evict(0, w, keep, 4, 8, to=to, to_weights=to_weights, kept=kept, workspace=space)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert np.array_equal(kept.cpu().numpy(), kept_rows(w.cpu().numpy(), keep, 4, 8))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        w.copy_(some_weights(hkv, length, 10 + i, "plain"))
        kept.zero_(), to_weights.zero_(), space.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        want = kept_rows(w.cpu().numpy(), keep, 4, 8)
        assert np.array_equal(kept.cpu().numpy(), want)
        assert torch.equal(to.view(0)[0].cpu(), torch.gather(k[0], 1, torch.from_numpy(want).long()[:, :, None].expand(-1, -1, d)))
        assert torch.equal(to_weights.cpu(), torch.gather(w.cpu(), 1, torch.from_numpy(want).long()))


def test_weigh_captured():
    cache, k, _ = filled(8, 2, 128, 700)
    q = draw((40, 8, 128), 5)
    lse = log_sum_exp(q, k[0], 128, 4).cuda()
    q, w = q.cuda(), torch.zeros((2, 700), device="cuda")
    cache.weigh(0, q, lse, w)
    torch.cuda.synchronize()
    once = w.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.weigh(0, q, lse, w)
    want = once
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = want + once
        assert torch.equal(w, want)


def test_a_fold_with_a_budget():
    """Chunks folded onto a cache that is cut down to its budget whenever it outgrows it, then carried on in 8 bits: steps, weights, eviction, append and the step on
    the 8-bit cache as a program has them.  Every step against attention in 64 bits over the rows that are kept."""
    import qcache_ref as R
    hq, hkv, d, n, budget = 8, 2, 64, 96, 160
    cache = kv.KvFoldCache(1, hq, hkv, d, n, budget + n)
    weights = torch.zeros((hkv, budget + n), device="cuda")
    rows = [torch.empty((hkv, 0, d), dtype=torch.bfloat16) for _ in range(2)]
    total = torch.zeros((hkv, 0), dtype=torch.float64)
    for chunk in range(5):
        q, k, v = (draw((n, h, d), 10 * chunk + i) for i, h in enumerate((hq, hkv, hkv)))
        prev = rows[0].shape[1]
        out, lse = torch.empty_like(q, device="cuda"), torch.empty((hq, n), device="cuda")
        cache.step(0, q.cuda(), k.cuda(), v.cuda(), out, lse=lse)
        cache.weigh(0, q.cuda(), lse, weights)
        rows = [torch.cat((old, new.transpose(0, 1)), 1) for old, new in zip(rows, (k, v))]
        ref, ref_lse, mean_abs, span = R.attend(q.double().numpy(), *(t.transpose(0, 1).double().numpy() for t in rows), prev, 1 / math.sqrt(d))
        assert np.abs(out.cpu().double().numpy() - ref).max() <= 2e-2
        w, tol = reference_weights(q, rows[0], lse.cpu(), d, hq // hkv)
        total = torch.cat((total, torch.zeros((hkv, n), dtype=torch.float64)), 1) + torch.from_numpy(w)
        got = weights[:, :prev + n].cpu()
        assert (got.double() - total).abs().max() < 1e-4 * n * (chunk + 1)
        total = got.double()
        if cache.length(0) > budget:
            kept = cache.evict(0, weights, budget, 4, 32, to_weights=weights).cpu()
            assert np.array_equal(kept.numpy(), kept_rows(got.numpy(), budget, 4, 32))
            index = kept.long()
            rows = [torch.gather(t, 1, index[:, :, None].expand(-1, -1, d)) for t in rows]
            total = torch.gather(total, 1, index)
    length = cache.length(0)
    small = kv.KvFoldQuantCache(1, hq, hkv, d, 8, length + 8)
    small.append(0, *(t[:, :length].transpose(0, 1) for t in cache.view(0)))
    q, k, v = (draw((3, h, d), 90 + i) for i, h in enumerate((hq, hkv, hkv)))
    out, lse = torch.empty_like(q, device="cuda"), torch.empty((hq, 3), device="cuda")
    small.step(0, q.cuda(), k.cuda(), v.cuda(), out, lse=lse)
    held = [R.held(torch.cat((t.transpose(0, 1), new)).float().numpy()) for t, new in zip(rows, (k, v))]
    ref, ref_lse, mean_abs, span = R.attend(q.double().numpy(), *held, length, 1 / math.sqrt(d))
    tol, tol_lse = R.bounds(ref, ref_lse, mean_abs, span, d, length + 3)
    assert (np.abs(out.cpu().double().numpy() - ref) <= tol).all() and (np.abs(lse.cpu().double().numpy() - ref_lse) <= tol_lse).all()


def test_refusals():
    cache, k, v = filled(8, 2, 64, 100, capacity=120, chunk=50, layers=2)
    w = torch.zeros((2, 120), device="cuda")
    q, lse = draw((10, 8, 64), 1).cuda(), torch.zeros((8, 10), device="cuda")
    status = lambda call: pytest.raises(kv.KvFoldError, call).value.status
    assert status(lambda: cache.weigh(2, q, lse, w)) == -2
    long = draw((51, 8, 64), 1).cuda()
    assert status(lambda: cache.weigh(0, long, torch.zeros((8, 51), device="cuda"), w)) == -1
    cache.truncate(1, 9)
    assert status(lambda: cache.weigh(1, q, lse, w)) == -3
    assert kv.kvfold_cache_weigh(cache.handle, 0, q.data_ptr(), 10, q.data_ptr(), None, lse.data_ptr(), w.data_ptr()) == -1
    assert kv.kvfold_cache_weigh(cache.handle, 0, q.data_ptr(), 10, None, None, lse.data_ptr(), w.data_ptr(), add=2) == -1
    assert kv.kvfold_cache_weigh(cache.handle, 0, q.data_ptr(), 10, None, None, w.data_ptr() + 4, w.data_ptr()) == -1  # one in the other
    assert kv.kvfold_cache_weigh(cache.handle, 0, q.data_ptr() + 2, 10, None, None, lse.data_ptr(), w.data_ptr()) == -1
    with pytest.raises(ValueError):
        cache.weigh(0, q, lse, w[:, :100])
    with pytest.raises(ValueError):
        cache.weigh(0, q.float(), lse, w)
    assert status(lambda: cache.evict(0, w, 0)) == -1
    assert status(lambda: cache.evict(0, w, 10, 5, 6)) == -1
    assert status(lambda: cache.evict(0, w, 10, -1, 0)) == -1
    assert status(lambda: cache.evict(0, w, 101)) == -3
    assert status(lambda: cache.evict(2, w, 10)) == -2
    small = kv.KvFoldCache(1, 8, 2, 64, 1, 9)
    assert status(lambda: cache.evict(0, w, 10, to=small)) == -4
    assert status(lambda: cache.evict(0, w, 10, to=kv.KvFoldCache(1, 8, 4, 64, 1, 20))) == -5
    assert status(lambda: cache.evict(0, w, 10, to=kv.KvFoldCache(1, 8, 2, 64, 1, 20, "f32"))) == -5
    assert status(lambda: cache.evict(0, w, 10, to=cache, to_layer=2)) == -2
    assert status(lambda: cache.evict(0, w, 10, workspace=torch.empty((16,), dtype=torch.uint8, device="cuda"))) == -6
    space = torch.empty((cache.evict_workspace_bytes(10),), dtype=torch.uint8, device="cuda")
    assert kv.kvfold_cache_evict(cache.handle, 0, w.data_ptr(), 10, 0, 0, None, 0, None, space.data_ptr(), space.data_ptr(), space.numel()) == -1
    assert kv.kvfold_cache_evict(cache.handle, 0, w.data_ptr(), 10, 0, 0, None, 0, None, w.data_ptr(), space.data_ptr(), space.numel()) == -1
    assert kv.kvfold_cache_evict(cache.handle, 0, w.data_ptr(), 10, 0, 0, None, 0, cache.view(0)[0].data_ptr(), None, space.data_ptr(), space.numel()) == -1
    assert cache.length(0) == 100
    with pytest.raises(ValueError):
        cache.evict(0, w, 10, kept=torch.empty((2, 9), dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("n", [1, 20])
def test_caches_whose_places_pass_32_bits(n):
    """Rows that are all alike, and 100 others behind them: 20 GB of rows, 160 MB of weights."""
    heads, d, same = 40, 128, 1_000_000
    length = same + 100
    cache = kv.KvFoldCache(1, heads, heads, d, 64, length + 28)
    first, tail = [draw((heads, 1, d), seed) for seed in (1, 2)], [draw((heads, 100, d), seed) for seed in (3, 4)]
    for view, x, y in zip(cache.view(0), first, tail):
        view[:, :same].copy_(x.cuda().expand(heads, same, d))
        view[:, same:length].copy_(y)
    cache.set_length(0, length)
    q, lse = draw((n, heads, d), 5), torch.full((heads, n), 14.0)
    weights = torch.full((heads, length + 28), 7.0, device="cuda")
    cache.weigh(0, q.cuda(), lse.cuda(), weights, add=False)
    want, tol = reference_weights(q, torch.cat((first[0], tail[0]), 1), lse, d, 1)
    got = torch.cat((weights[:, :1], weights[:, same:length]), 1).cpu().double().numpy()
    assert (np.abs(got - want) <= tol).all()
    assert (weights[:, :same] == weights[:, :1]).all() and (weights[:, length:] == 7).all()
    order = torch.sort(weights[:, 4:length - 10], dim=1, descending=True, stable=True).indices[:, :66] + 4
    ends = torch.cat((torch.arange(4), torch.arange(length - 10, length))).cuda().expand(heads, 14)
    expected = torch.sort(torch.cat((order, ends), 1), dim=1).values
    rows = [torch.gather(view, 1, expected[:, :, None].expand(heads, 80, d)) for view in cache.view(0)]
    for to in (kv.KvFoldCache(1, heads, heads, d, 64, 100), None):
        kept = torch.empty((heads, 80), dtype=torch.int32, device="cuda")
        cache.evict(0, weights, 80, 4, 10, to=to, kept=kept)
        assert torch.equal(kept.long(), expected)
        for view, x in zip((to or cache).view(0), rows):
            assert torch.equal(view[:, :80], x)
    assert cache.length(0) == 80


def test_kept_weights_lie_on_the_weights_or_apart():
    cache, _, _ = filled(4, 2, 64, 100)
    w = torch.rand((2 * 100 + 50,), device="cuda")
    space = torch.empty((cache.evict_workspace_bytes(60),), dtype=torch.uint8, device="cuda")
    call = lambda to: kv.kvfold_cache_evict(cache.handle, 0, w.data_ptr(), 60, 0, 0, None, 0, to, None, space.data_ptr(), space.numel())
    assert call(w.data_ptr() + 4) == -1 and call(w.data_ptr() + 4 * 50) == -1 and cache.length(0) == 100
    assert call(w.data_ptr()) == 0 and cache.length(0) == 60
