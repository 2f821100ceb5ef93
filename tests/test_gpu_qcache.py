"""The cache held in 8 bits on the GPU against its definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2605_12471_amd as kv
from paper_2605_12471_amd import inputs as I
import qcache_ref as R

pytestmark = pytest.mark.gpu
SHAPES = [(4, 1, 64), (8, 2, 128), (7, 1, 128), (3, 3, 64), (40, 2, 64), (6, 6, 128)]  # query heads, KV heads, head dim


def draw(shape, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * gain).to(torch.bfloat16)


def rotated(x, cos, sin):
    """The rotary step's arithmetic: the product with the sine rounded to fp32, the rest exact, rounded to fp32, then to bf16."""
    half = x.shape[-1] // 2
    lo, up, c, s = x[..., :half].double(), x[..., half:].double(), cos[:, None].double(), sin[:, None].double()
    return torch.cat(((lo * c - (up * s).float().double()).float(), (up * c + (lo * s).float().double()).float()), -1).to(torch.bfloat16)


class Fold:
    """A cache and what it has to hold."""

    def __init__(self, hq, hkv, d, capacity, seed=0, chunk=None, layers=1):
        self.hq, self.hkv, self.d, self.seed = hq, hkv, d, seed
        self.cache = kv.KvFoldQuantCache(layers, hq, hkv, d, chunk or capacity, capacity)
        self.k, self.v = (torch.empty((0, hkv, d), dtype=torch.bfloat16) for _ in range(2))

    def chunk(self, n, gain=1.0):
        self.seed += 3
        return draw((n, self.hq, self.d), self.seed), draw((n, self.hkv, self.d), self.seed + 1, gain), draw((n, self.hkv, self.d), self.seed + 2)

    def joined(self, k, v):
        self.k, self.v = torch.cat((self.k, k)), torch.cat((self.v, v))

    def append(self, n):
        _, k, v = self.chunk(n)
        self.cache.append(0, k.cuda(), v.cuda())
        self.joined(k, v)

    def step(self, n, rope=False, data=None, stream=None):
        q, k, v = data or self.chunk(n)
        prev = len(self.k)
        angles = I.rope_tables(self.d, prev, n) if rope else None
        out, lse = torch.full((n, self.hq, self.d), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((self.hq, n), float("nan"), device="cuda")
        self.cache.step(0, q.cuda(), k.cuda(), v.cuda(), out, lse=lse, rope=tuple(t.cuda() for t in angles) if rope else None, stream=stream)
        if rope:
            q, k = rotated(q, *angles), rotated(k, *angles)
        self.joined(k, v)
        self.check(q, prev, out, lse)
        return out, lse

    def held(self):
        return R.held(self.k.float().numpy()), R.held(self.v.float().numpy())

    def check(self, q, prev, out, lse):
        k, v = self.held()
        n = len(q)
        assert self.cache.length(0) == prev + n == len(k)
        ref, ref_lse, mean_abs, span = R.attend(q.double().numpy(), k[:prev + n], v[:prev + n], prev, 1 / math.sqrt(self.d))
        tol, tol_lse = R.bounds(ref, ref_lse, mean_abs, span, self.d, prev + n)
        err, err_lse = np.abs(out.cpu().double().numpy() - ref), np.abs(lse.cpu().double().numpy() - ref_lse)
        for got, want, e, t in ((out, ref, err, tol), (lse, ref_lse, err_lse, tol_lse)):
            bad = np.argwhere(~(e <= t))
            assert not len(bad), [(tuple(i), float(got[tuple(i)]), want[tuple(i)], e[tuple(i)], t[tuple(i)]) for i in bad[:5]] + [len(bad)]

    def check_rows(self, first=0):
        n = len(self.k) - first
        got = [torch.full((n, self.hkv, self.d), float("nan"), device="cuda") for _ in range(2)]
        self.cache.read(0, first, *got)
        for x, ref in zip(got, self.held()):
            assert np.array_equal(x.cpu().numpy(), ref[first:].astype(np.float32))


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("sizes", [[1], [63, 1, 1], [64, 64], [1, 127, 3], [200, 1, 70], [50, 200, 6]])
def test_fold_and_rows(hq, hkv, d, sizes):
    f = Fold(hq, hkv, d, sum(sizes) + 5, seed=sum(sizes))
    for n in sizes:
        f.step(n)
        f.check_rows()


@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("prev", [0, 1, 62, 63, 64, 129, 1000, 4187])
@pytest.mark.parametrize("n", [1, 2, 4, 17, 65])
def test_steps_on_caches_of_any_length(hq, hkv, d, prev, n):
    f = Fold(hq, hkv, d, prev + n, seed=prev + n)
    f.append(prev)
    f.step(n)
    f.check_rows()


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (28, 4, 128), (32, 8, 64)])
@pytest.mark.parametrize("prev,n", [(20000, 1), (9001, 3), (8000, 37), (3000, 300), (0, 700)])
def test_sizes_of_a_model(hq, hkv, d, prev, n):
    f = Fold(hq, hkv, d, prev + n, seed=prev + n)
    f.append(prev)
    f.step(n)


@pytest.mark.parametrize("hq,hkv,d", SHAPES[:4])
@pytest.mark.parametrize("prev,n", [(0, 5), (60, 9), (130, 1), (100, 150)])
def test_rotary_embedding_in_the_step(hq, hkv, d, prev, n):
    f = Fold(hq, hkv, d, prev + n, seed=n)
    f.append(prev)
    f.step(n, rope=True)
    f.check_rows()


def test_what_is_held_does_not_depend_on_the_chunks():
    rows = []
    for sizes in ([300], [1] * 3 + [100, 61, 136], [64, 64, 172]):
        f = Fold(8, 2, 128, 300)
        k, v = draw((300, 2, 128), 1), draw((300, 2, 128), 2)
        at = 0
        for n in sizes:
            f.cache.append(0, k[at:at + n].cuda(), v[at:at + n].cuda())
            at += n
        got = [torch.empty((300, 2, 128), device="cuda") for _ in range(2)]
        f.cache.read(0, 0, *got)
        rows.append(torch.stack(got))
    assert torch.equal(rows[0], rows[1]) and torch.equal(rows[0], rows[2])


def test_append_of_a_caches_own_rows():
    """A layer folded in bf16 goes on in 8 bits: the rows as they lie, head by head."""
    n, hkv, d = 200, 4, 64
    with kv.KvFoldCache(1, 8, hkv, d, n, n + 50) as cache:
        k, v = draw((n, hkv, d), 1), draw((n, hkv, d), 2)
        out = torch.empty((n, 8, d), dtype=torch.bfloat16, device="cuda")
        cache.step(0, draw((n, 8, d), 3).cuda(), k.cuda(), v.cuda(), out)
        f = Fold(8, hkv, d, n + 10)
        f.cache.append(0, *(t[:, :n].transpose(0, 1) for t in cache.view(0)))
        torch.cuda.synchronize()
    f.joined(k, v)
    f.check_rows()
    f.step(3)


@pytest.mark.parametrize("d", [64, 128])
def test_numbers_that_are_hard_to_hold(d):
    """Zero blocks, tiny ones, the largest, one large element among small ones, halves between codes, infinities and NaN."""
    n, hkv = 64 * 7 + 9, 2
    f = Fold(4, hkv, d, n + 1)
    q, k, v = f.chunk(n)
    for x in (k, v):
        x[:64] = 0
        x[64:128] *= 1e-36
        x[128:192] *= 2.0 ** 100
        x[192:256, 0, 0] = 1000
        x[256:320] = torch.randint(-127, 128, (64, hkv, d)).to(torch.bfloat16) / 2
        x[256, :, 0] = 127
        x[320, 0, 1], x[321, 0, 1], x[322, 0, 1] = math.inf, -math.inf, math.nan
        x[-2, 0, 3], x[-1, 1, 4] = math.inf, math.nan
    f.cache.append(0, k.cuda(), v.cuda())
    f.joined(k, v)
    f.check_rows()


@pytest.mark.parametrize("prev,n", [(10, 4), (10, 40), (100, 200)])
def test_rows_do_not_take_harm_from_what_they_do_not_see(prev, n):
    """The chunk's last token is not finite: the rows before it see nothing of it (but a block that holds it takes its scales from it)."""
    f = Fold(8, 2, 128, prev + n)
    f.append(prev)
    q, k, v = f.chunk(n)
    k[-1], v[-1] = math.inf, math.nan
    v[-1, 0, 0] = -math.inf
    out = torch.empty((n, 8, 128), dtype=torch.bfloat16, device="cuda")
    f.cache.step(0, q.cuda(), k.cuda(), v.cuda(), out)
    f.joined(k, v)
    kk, vv = f.held()
    ref, ref_lse, mean_abs, span = R.attend(q.double().numpy()[:n - 1], kk[:-1], vv[:-1], prev, 1 / math.sqrt(128))
    tol, _ = R.bounds(ref, ref_lse, mean_abs, span, 128, prev + n)
    assert (np.abs(out[:n - 1].cpu().double().numpy() - ref) <= tol).all()


@pytest.mark.parametrize("profile", ["step20", "step100", "stairs", "spike", "deep_start"])
@pytest.mark.parametrize("n", [1, 20, 300])
def test_logits_that_jump(profile, n):
    cfg = I.FoldConfig("t", 77, 1, 8, 2, 64, 400, 700, "bf16")
    f = Fold(8, 2, 64, 700)
    for at, m in ((0, 400), (400, n)):
        q, k, v = I.steered_qkv(cfg, 0, 0, profile, n_tokens=m, token_base=at)
        f.step(m, data=(q, k, v))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("profile", [lambda j: 45.0 * (j >= 500), lambda j: 60.0 * (j >= 1100), lambda j: 100.0 * ((j >= 300) + (j >= 900)), lambda j: 0.4 * j,
                                     lambda j: 90.0 * (j == 700), lambda j: -200.0 * (j < 130), lambda j: 80.0 * (j >= 1550)])
def test_logits_that_jump_far_behind_a_piece_s_first_block(d, profile):
    """Jumps of 2^65 and more between blocks of a piece (many rows, so that pieces are long): the reference follows, or the piece is done again."""
    hq, hkv, prev, n = 16, 8, 1400, 1000
    f = Fold(hq, hkv, d, prev + n)
    g = torch.Generator().manual_seed(d)
    u = torch.nn.functional.normalize(torch.randn(d, generator=g), dim=0)
    level = torch.tensor([float(profile(j)) for j in range(prev + n)])
    k = (0.1 * torch.randn((prev + n, hkv, d), generator=g) + 0.5 * level[:, None, None] * u).to(torch.bfloat16)
    v = torch.randn((prev + n, hkv, d), generator=g).to(torch.bfloat16)
    q = (0.1 * torch.randn((n, hq, d), generator=g) + 2 * math.sqrt(d) * u).to(torch.bfloat16)
    f.cache.append(0, k[:prev].cuda(), v[:prev].cuda())
    f.joined(k[:prev], v[:prev])
    f.step(n, data=(q, k[prev:], v[prev:]))


def test_rewinding():
    f = Fold(8, 2, 128, 1000)
    f.append(500)
    f.step(1)
    for back in (3, 40, 52):  # to 449 at the least: block 7 begins at 448, block 6 at 384
        n = len(f.k) - back
        f.cache.truncate(0, n)
        f.k, f.v = f.k[:n], f.v[:n]
        f.check_rows()
        f.step(2)
    f.cache.truncate(-1, 128)
    f.k, f.v = f.k[:128], f.v[:128]
    f.check_rows()
    f.step(70)
    f.step(1)
    f.check_rows()


def test_rewinding_as_far_as_the_rows_are_there():
    f = Fold(4, 1, 64, 1000)
    f.append(300)                      # blocks 3 and 4 in bf16
    for n in (191, 1, 130):
        with pytest.raises(kv.KvFoldError) as e:
            f.cache.truncate(0, n)
        assert e.value.status == -3
    assert f.cache.length(0) == 300
    f.cache.truncate(0, 193)
    f.k, f.v = f.k[:193], f.v[:193]
    f.step(200)                        # 393: blocks 5 and 6
    with pytest.raises(kv.KvFoldError):
        f.cache.truncate(0, 319)
    f.cache.truncate(0, 321)
    f.k, f.v = f.k[:321], f.v[:321]
    f.check_rows()
    f.cache.truncate(0, 0)
    f.k, f.v = f.k[:0], f.v[:0]
    f.step(5)


def test_layers_and_caches_are_apart():
    a, b = kv.KvFoldQuantCache(2, 4, 2, 64, 100, 200), kv.KvFoldQuantCache(1, 4, 2, 64, 100, 200)
    data = [(draw((90, 4, 64), s), draw((90, 2, 64), s + 1), draw((90, 2, 64), s + 2)) for s in (1, 11, 21)]
    outs = []
    for cache, layer, (q, k, v) in ((a, 0, data[0]), (a, 1, data[1]), (b, 0, data[2])):
        cache.step(layer, q.cuda(), k.cuda(), v.cuda(), torch.empty_like(q, device="cuda"))
    for cache, layer, (q, k, v) in ((a, 0, data[0]), (a, 1, data[1]), (b, 0, data[2])):
        got = [torch.empty((90, 2, 64), device="cuda") for _ in range(2)]
        cache.read(layer, 0, *got)
        for x, rows in zip(got, (k, v)):
            assert np.array_equal(x.cpu().numpy(), R.held(rows.float().numpy()).astype(np.float32))


@pytest.mark.parametrize("n,prev", [(1, 3000), (40, 500), (1, 63)])
def test_same_bits_every_time_and_on_another_stream(n, prev):
    f = Fold(32, 8, 128, prev + n)
    f.append(prev)
    data = f.chunk(n)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = []
    for i in range(6):
        f.cache.truncate(0, prev)
        f.k, f.v = f.k[:prev], f.v[:prev]
        with torch.cuda.stream(side if i % 2 else torch.cuda.default_stream()):
            got.append(f.step(n, data=data))
        torch.cuda.synchronize()
    assert all(torch.equal(o, got[0][0]) and torch.equal(l, got[0][1]) for o, l in got)


@pytest.mark.parametrize("n,prev", [(1, 5000), (30, 700), (300, 256)])
def test_captured_step(n, prev):
    f = Fold(8, 2, 128, prev + n)
    f.append(prev)
    q, k, v = (t.cuda() for t in f.chunk(n))
    out, lse = torch.empty_like(q), torch.empty((8, n), device="cuda")

    def step():
        f.cache.truncate(0, prev)
        f.cache.step(0, q, k, v, out, lse=lse)

    step()
    torch.cuda.synchronize()
    want = out.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        out.zero_(), lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        q.copy_(torch.roll(q, 1, 0)) if i == 1 else None
        if i == 1:
            step()
            torch.cuda.synchronize()
            want = out.clone(), lse.clone()


@pytest.mark.parametrize("n,prev", [(2, 900), (50, 100), (200, 64)])
def test_output_in_the_place_of_an_input(n, prev):
    f = Fold(4, 4, 64, prev + n)
    f.append(prev)
    q, k, v = f.chunk(n)
    want, _ = f.step(n, data=(q, k, v))
    for name in ("q", "k", "v"):
        t = {"q": q.cuda(), "k": k.cuda(), "v": v.cuda()}
        f.cache.truncate(0, prev)
        f.cache.step(0, t["q"], t["k"], t["v"], t[name])
        assert torch.equal(t[name], want)


def test_memory_around_the_results_is_left_alone():
    n, prev = 37, 100
    f = Fold(8, 2, 128, prev + n)
    f.append(prev)
    q, k, v = f.chunk(n)
    out = torch.full((n + 20, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((8 * n + 20,), 7.0, device="cuda")
    f.cache.step(0, q.cuda(), k.cuda(), v.cuda(), out[:n], lse=lse[:8 * n].view(8, n))
    rows = torch.full((n + 4, 2, 128), 7.0, device="cuda")
    f.cache.read(0, 100, rows[:n], None)
    assert (out[n:] == 7).all() and (lse[8 * n:] == 7).all() and (rows[n:] == 7).all()


def test_storage_of_the_callers():
    import ctypes
    from paper_2605_12471_amd import binding
    cfg = binding.make_config(1, 4, 2, 64, 64, 200, kv.KVFOLD_BF16)
    need = kv.kvfold_qcache_bytes_required(cfg)
    buf = torch.full((need + 512,), 0xff, dtype=torch.uint8, device="cuda")
    base = (buf.data_ptr() + 255) // 256 * 256
    cfg.kv_buffer, cfg.kv_buffer_bytes = base, need
    rc, h = kv.kvfold_qcache_create(cfg)
    assert rc == 0
    k = draw((130, 2, 64), 1).cuda()
    assert kv.kvfold_qcache_append(h, 0, k.data_ptr(), k.data_ptr(), 128, 64, 130, 0) == 0
    got = torch.empty((130, 2, 64), device="cuda")
    assert kv.kvfold_qcache_read(h, 0, 0, 130, got.data_ptr(), None) == 0
    torch.cuda.synchronize()
    assert np.array_equal(got.cpu().numpy(), R.held(k.float().cpu().numpy()).astype(np.float32))
    q = draw((1, 4, 64), 5).cuda()
    out = torch.empty_like(q)
    assert kv.kvfold_qcache_step(h, 0, q.data_ptr(), k.data_ptr(), k.data_ptr(), 1, 130, None, None, base, None) == -1  # the output on the cache
    assert kv.kvfold_qcache_step(h, 0, q.data_ptr(), k.data_ptr(), k.data_ptr(), 1, 130, None, None, out.data_ptr(), q.data_ptr()) == -1
    assert kv.kvfold_qcache_destroy(h) == 0
    off = base - buf.data_ptr()
    assert (buf[:off] == 0xff).all() and (buf[off + need:] == 0xff).all()


def test_refusals():
    f = Fold(8, 2, 64, 100, chunk=50)
    q, k, v = (t.cuda() for t in f.chunk(50))
    out = torch.empty_like(q)
    status = lambda call: pytest.raises(kv.KvFoldError, call).value.status
    assert status(lambda: f.cache.step(1, q, k, v, out)) == -2
    assert status(lambda: f.cache.step(0, q, k, v, out, pos_offset=1)) == -3
    q2, k2, v2 = (t.cuda() for t in f.chunk(51))
    assert status(lambda: f.cache.step(0, q2, k2, v2, torch.empty_like(q2))) == -1  # more than a chunk
    f.cache.append(0, k, v)
    f.cache.append(0, k[:20], v[:20])
    assert status(lambda: f.cache.step(0, q, k, v, out)) == -4
    assert status(lambda: f.cache.append(0, k, v)) == -4
    assert status(lambda: f.cache.read(0, 60, torch.empty((11, 2, 64), device="cuda"), None)) == -3
    assert status(lambda: f.cache.truncate(0, 71)) == -3
    rope = tuple(t.cuda() for t in I.rope_tables(64, 70, 4))
    assert kv.kvfold_qcache_step(f.cache.handle, 0, q.data_ptr(), k.data_ptr(), v.data_ptr(), 4, 70, rope[0].data_ptr(), None, out.data_ptr()) == -1
    assert kv.kvfold_qcache_step(f.cache.handle, 0, q.data_ptr(), k.data_ptr(), v.data_ptr(), 4, 70, None, None, q.data_ptr() + 64) == -1  # not in q's place
    assert kv.kvfold_qcache_append(f.cache.handle, 0, k.data_ptr(), v.data_ptr(), 129, 64, 4, 70) == -1
    assert f.cache.length(0) == 70
    for bad in (dict(q=q.float()), dict(k_new=k[:49]), dict(v_new=v.cpu()), dict(out=out.transpose(0, 1)), dict(lse=torch.empty((8, 49), device="cuda"))):
        args = {"q": q, "k_new": k, "v_new": v, "out": out, **bad}
        with pytest.raises(ValueError):
            f.cache.step(0, args["q"], args["k_new"], args["v_new"], args["out"], lse=args.get("lse"))
    with pytest.raises(ValueError):
        f.cache.append(0, k, v.transpose(0, 1).contiguous().transpose(0, 1))
    f.cache.append(0, k[:0], v[:0])
    assert f.cache.length(0) == 70


@pytest.mark.parametrize("hq,hkv,d,same", [(40, 40, 128, 1_000_000), (4, 1, 64, 33_554_240)])
@pytest.mark.parametrize("n", [1, 20])
def test_caches_whose_places_pass_32_bits(hq, hkv, d, same, n):
    """Rows that are all alike, 5 GB of codes or 2 GiB of a head's, and 60 + n others behind them, which get the larger part of the weight."""
    cache = kv.KvFoldQuantCache(1, hq, hkv, d, 64, same + 128)
    first = [draw((1, hkv, d), seed) for seed in (1, 2)]
    cache.append(0, *(x.cuda().expand(same, hkv, d) for x in first))
    tail = [draw((60 + n, hkv, d), seed) for seed in (3, 4)]
    cache.append(0, *(x[:60].cuda() for x in tail))
    q = draw((n, hq, d), 5, 6.0)
    out, lse = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((hq, n), device="cuda")
    cache.step(0, q.cuda(), *(x[60:].cuda() for x in tail), out, lse=lse)
    assert cache.length(0) == same + 60 + n
    one = [R.held(x.expand(64, hkv, d).float().numpy())[:1] for x in first]
    others = [R.held(x.float().numpy()) for x in tail]
    for begin, ref in ((0, one), (same // 2 + 5, one), (same - 1, [np.concatenate(x) for x in zip(one, others)])):
        got = [torch.empty(ref[0].shape, device="cuda") for _ in range(2)]
        cache.read(0, begin, *got)
        for x, y in zip(got, ref):
            assert np.array_equal(x.cpu().numpy(), y.astype(np.float32))
    k, v = (np.concatenate(x) for x in zip(one, others))
    seen = np.arange(61 + n)[None, :] <= 61 + np.arange(n)[:, None]
    times = np.where(np.arange(61 + n) == 0, float(same), 1.0)
    ref, mean_abs, ref_lse, span = np.empty((n, hq, d)), np.empty((n, hq, d)), np.empty((hq, n)), np.empty((hq, n))
    for h in range(hq):
        g, qq = h // (hq // hkv), q[:, h].double().numpy()
        s, a = qq @ k[:, g].T / math.sqrt(d), np.abs(qq) @ np.abs(k[:, g]).T / math.sqrt(d)
        top = np.where(seen, s, -np.inf).max(-1, keepdims=True)
        p = np.where(seen, times * np.exp(s - top), 0)
        total = p.sum(-1, keepdims=True)
        ref_lse[h], span[h] = (top + np.log(total))[:, 0], np.where(seen, a, 0).max(-1)
        ref[:, h], mean_abs[:, h] = p / total @ v[:, g], p / total @ np.abs(v[:, g])
    tol, tol_lse = R.bounds(ref, ref_lse, mean_abs, span, d, same + 60 + n)
    assert (np.abs(out.cpu().double().numpy() - ref) <= tol).all() and (np.abs(lse.cpu().double().numpy() - ref_lse) <= tol_lse).all()


@pytest.mark.parametrize("prev,n", [(24_010, 65), (24_640, 130)])
def test_eight_wavefronts_64_wide(prev, n):
    f = Fold(40, 2, 64, prev + n, seed=9)
    f.append(prev)
    f.step(n)
    f.check_rows(first=prev - 70)


@pytest.mark.parametrize("prev", [0, 64, 128, 100])
@pytest.mark.parametrize("n", [64, 65, 128, 130, 192, 193, 256, 300])
def test_rows_taken_back_behind_a_chunk(prev, n):
    """The last blocks' rows are in bf16 wherever the chunk began."""
    f = Fold(8, 2, 128, prev + n + 64, seed=prev + n)
    f.append(prev)
    f.append(n)
    for back in (1, 37, 64):
        f.cache.truncate(0, prev + n - back)
        f.k, f.v = f.k[:prev + n - back], f.v[:prev + n - back]
        f.check_rows()
        f.append(back)
    f.step(2)
    f.check_rows()


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (32, 8, 64), (28, 4, 128), (40, 2, 64)])
@pytest.mark.parametrize("prev,n", [(0, 17), (64, 63), (1000, 20), (4187, 32), (4160, 37)])
@pytest.mark.parametrize("rope", [False, True])
def test_chunks_that_fill_no_block(hq, hkv, d, prev, n, rope):
    f = Fold(hq, hkv, d, prev + n + 70, seed=prev + n)
    f.append(prev)
    f.step(n, rope=rope)
    f.check_rows(first=max(0, prev - 70))
    f.append(70)                       # the block is filled from what the step has left
    f.check_rows(first=max(0, prev - 70))


def test_a_chunk_that_fills_no_block_captured():
    """Rows, queries and results of another replay, the cache's ring written by each."""
    f = Fold(8, 2, 128, 600, seed=4)
    f.append(500)
    data = [f.chunk(10) for _ in range(3)]
    q, k, v = (x.cuda() for x in data[0])
    out = torch.empty_like(q)
    f.cache.step(0, q, k, v, out)
    f.cache.truncate(0, 500)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f.cache.step(0, q, k, v, out)
    for x, y, z in data + data:
        q.copy_(x), k.copy_(y), v.copy_(z)
        graph.replay()
        got = out.clone()
        f.cache.truncate(0, 500)
        again = torch.empty_like(out)
        f.cache.step(0, q, k, v, again)
        torch.cuda.synchronize()
        assert torch.equal(got, again)


@pytest.mark.parametrize("prev,n", [(3000, 1), (3000, 3), (2000, 40), (2048, 200)])
def test_two_caches_on_two_streams(prev, n):
    """Steps that run beside each other, pieces and their meeting included, leave the bits of steps one after the other."""
    folds = [Fold(16, 4, 128, prev + n, seed=s) for s in (1, 50)]
    data, want, got = [], [], []
    for f in folds:
        f.append(prev)
        data.append([x.cuda() for x in f.chunk(n)])
        q, k, v = data[-1]
        want.append(f.cache.step(0, q, k, v, torch.empty_like(q)))
        f.cache.truncate(0, prev)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in folds]
    for _ in range(10):
        for f, (q, k, v), s in zip(folds, data, streams):
            with torch.cuda.stream(s):
                got.append(f.cache.step(0, q, k, v, torch.empty_like(q)))
            f.cache.truncate(0, prev)
    torch.cuda.synchronize()
    assert all(torch.equal(x, want[i % 2]) for i, x in enumerate(got))
