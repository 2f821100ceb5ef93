"""The cache in pages on the GPU against its definition in 64 bits: places of new tokens, decoding, prompts and chunks of them."""
import math

import numpy as np
import pytest
import torch

import paper_2605_12471_amd as kv
import pcache_ref as R

pytestmark = pytest.mark.gpu
SHAPES = [(4, 1, 64), (8, 2, 128), (7, 1, 128), (3, 3, 64), (40, 2, 64), (6, 6, 128)]  # query heads, KV heads, head dim


def draw(gen, shape, dtype, gain=1.0):
    return (torch.randn(shape, generator=gen) * gain).to(R.TYPE[dtype])


class Fold:
    """A batch on a cache whose every row that no sequence has is NaN."""

    def __init__(self, hq, hkv, d, page, prev, new, dtype="bf16", seed=0, pad=0, spare=3, layers=1, fused=False, one_each=False, max_new=None, max_len=None, layer=0,
                 holes=(), present=False, width=0, lead=0):
        self.hq, self.hkv, self.d, self.page, self.prev, self.new, self.dtype, self.layer = hq, hkv, d, page, list(prev), list(new), dtype, layer
        g = torch.Generator().manual_seed(seed + 977 * sum(prev) + sum(new))
        counts = [-(-(p + n) // page) for p, n in zip(prev, new)]
        self.n_pages = sum(counts) + spare
        self.cache = kv.KvFoldPagedCache(layers, hq, hkv, d, page, self.n_pages, dtype)
        order = torch.randperm(self.n_pages, generator=g).tolist()
        width = max(counts + [1, width - 2]) + 2
        self.tables = torch.full((len(prev), width), -7, dtype=torch.int32)
        self.rows, self.n_tokens, self.lead = lead + sum(new) + pad, lead + sum(new), lead
        self.slots = torch.full((self.rows,), -1, dtype=torch.int64)
        shape = (self.n_pages, hkv, page, d)
        self.k_pages, self.v_pages = (torch.full(shape, math.nan, dtype=R.TYPE[dtype]) for _ in range(2))
        self.k, self.v, at, self.cu = [], [], lead, [lead]
        if fused:
            together = draw(g, (self.rows, (hq + 2 * hkv) * d), dtype).cuda()
            self.dev = [t.unflatten(1, (-1, d)) for t in together.split((hq * d, hkv * d, hkv * d), 1)]
        else:
            self.dev = [draw(g, (self.rows, heads, d), dtype).cuda() for heads in (hq, hkv, hkv)]
        self.q, self.kn, self.vn = (t.cpu() for t in self.dev)
        for s, (p, n) in enumerate(zip(prev, new)):
            for j in range(counts[s]):
                self.tables[s, j] = order.pop()
            old = [draw(g, (p, hkv, d), dtype) for _ in range(2)]
            where = torch.arange(p + n)
            numbers = self.tables[s, where // page].long()
            if present:  # the new rows are there already
                old = [torch.cat((o, x[at:at + n])) for o, x in zip(old, (self.kn, self.vn))]
            for pages, rows in ((self.k_pages, old[0]), (self.v_pages, old[1])):
                pages[numbers[:len(rows)], :, (where % page)[:len(rows)]] = rows
            self.slots[at:at + n] = (numbers * page + where % page)[p:]
            self.k.append(torch.cat((old[0][:p], self.kn[at:at + n])))
            self.v.append(torch.cat((old[1][:p], self.vn[at:at + n])))
            at += n
            self.cu.append(at)
        self.present = present
        self.hidden = {}
        for s, j in holes:  # pages that the table does not name
            self.hidden.setdefault(s, []).append(j)
            self.tables[s, j] = (-1, 1 << 30, self.n_pages)[(s + j) % 3]
        for pages, rows in zip(self.cache.view(layer), (self.k_pages, self.v_pages)):
            pages.copy_(rows)
        self.batch = kv.KvFoldBatch(self.cache, self.tables.cuda(), self.rows, max_new or max(list(new) + [1]),
                                    max_len or max([p + n for p, n in zip(prev, new)] + [1]),
                                    lens=torch.tensor([p + n for p, n in zip(prev, new)], dtype=torch.int32).cuda(),
                                    cu_new=torch.tensor(self.cu, dtype=torch.int32).cuda(), slots=self.slots.cuda(), one_each=one_each)

    def step(self, stream=None):
        self.out = torch.full((self.rows, self.hq, self.d), 77.0, dtype=R.TYPE[self.dtype], device="cuda")
        self.lse = torch.full((self.hq, self.rows), 77.0, device="cuda")
        k, v = (None, None) if self.present else self.dev[1:]
        self.cache.step(self.layer, self.batch, self.dev[0], k, v, self.out, lse=self.lse, stream=stream)
        return self

    def visible(self, s):
        p, n = self.prev[s], self.new[s]
        seen = np.arange(p + n)[None, :] <= p + np.arange(n)[:, None]
        for j in self.hidden.get(s, ()):
            seen[:, j * self.page:(j + 1) * self.page] = False
        return seen

    def check(self, rows=None):
        """Against the definition; rows: of each sequence only the first so many of its new ones."""
        out, lse = self.out.cpu(), self.lse.cpu().double().numpy()
        for s, n in enumerate(self.new if rows is None else rows):
            first, seen = self.cu[s], self.visible(s)[:n]
            k, v = self.k[s].clone(), self.v[s].clone()
            hidden = torch.tensor(~seen.any(0))
            k[hidden], v[hidden] = 0, 0
            ref, ref_lse, mean_abs, span = R.attend(self.q[first:first + n], k, v, seen, 1 / math.sqrt(self.d))
            tol, tol_lse = R.bounds(ref, ref_lse, mean_abs, span, self.d, len(k), self.dtype)
            for name, got, want, t in (("out", out[first:first + n].double().numpy(), ref, tol), ("lse", lse[:, first:first + n], ref_lse, tol_lse)):
                with np.errstate(invalid="ignore"):
                    bad = np.argwhere(~((np.abs(got - want) <= t) | (got == want)))
                assert not len(bad), (name, s, self.prev[s], n, len(bad), [(tuple(i), got[tuple(i)], want[tuple(i)], t[tuple(i)]) for i in bad[:4]])
        assert (out[self.n_tokens:] == 77).all() and (lse[:, self.n_tokens:] == 77).all() and (out[:self.lead] == 77).all() and (lse[:, :self.lead] == 77).all()
        return self

    def check_pages(self):
        """The new rows at their places, everything else as it was."""
        for got, want, new in zip(self.cache.view(self.layer), (self.k_pages, self.v_pages), (self.kn, self.vn)):
            want = want.clone()
            slots = self.slots[self.lead:self.n_tokens]
            want[slots // self.page, :, slots % self.page] = new[self.lead:self.n_tokens]
            view = torch.int16 if self.dtype == "bf16" else torch.int32
            assert torch.equal(got.cpu().view(view), want.view(view))
        return self


DECODE = [([0], [1]), ([15], [1]), ([16], [1]), ([300], [1]), ([1, 0, 31, 32, 33, 127, 128, 700], [1] * 8), ([5, 640, 0, 17], [0, 1, 0, 1]),
          ([2000, 3, 129, 4187], [1] * 4), ([9000], [1])]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", SHAPES[:4] + SHAPES[5:])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("prev,new", DECODE)
def test_decoding(hq, hkv, d, page, prev, new, dtype):
    Fold(hq, hkv, d, page, prev, new, dtype).step().check().check_pages()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,new", [(4, 1, 64, [4, 3, 0, 1, 4]), (8, 2, 128, [4, 4, 2, 1, 3]), (3, 3, 64, [16, 5, 9, 16, 1]), (7, 1, 128, [2, 1, 2, 2, 2])])
@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("prev", [[0, 14, 30, 60, 1000], [28, 31, 0, 16, 17], [126, 127, 125, 4100, 64]])
def test_a_few_tokens_of_every_sequence(hq, hkv, d, new, page, prev, dtype):
    Fold(hq, hkv, d, page, prev, new, dtype, pad=3).step().check().check_pages()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("prev,new", [([0], [17]), ([0, 0, 0], [64, 1, 200]), ([63, 64, 65, 0, 3], [65, 33, 0, 1, 130]), ([0, 500], [300, 40]), ([1000], [33])])
def test_prompts_and_chunks(hq, hkv, d, page, prev, new, dtype):
    Fold(hq, hkv, d, page, prev, new, dtype).step().check().check_pages()


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 32, 8, 128), ("bf16", 28, 4, 128), ("bf16", 32, 8, 64), ("f32", 8, 2, 128)])
@pytest.mark.parametrize("prev,new,page", [([20000], [1], 128), ([9000, 100], [3, 2], 16), ([8000, 11], [37, 300], 64), ([0, 0, 5], [700, 1, 129], 32),
                                           ([3000, 2500, 4000], [64, 64, 64], 64)])
def test_sizes_of_a_model(dtype, hq, hkv, d, prev, new, page):
    Fold(hq, hkv, d, page, prev, new, dtype, fused=True, pad=5).step().check().check_pages()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (40, 2, 64), (18, 1, 64)])
def test_one_token_of_each_without_a_running_sum(hq, hkv, d, dtype):
    """(also where so many heads share a KV head that it is a prompt's kernel)"""
    f = Fold(hq, hkv, d, 32, [0, 5, 300, 64, 1], [1] * 5, dtype, one_each=True).step().check().check_pages()
    g = Fold(hq, hkv, d, 32, [0, 5, 300, 64, 1], [1] * 5, dtype).step()
    assert torch.equal(f.out, g.out) and torch.equal(f.lse, g.lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prev,new", [([40, 0, 700], [1, 1, 1]), ([40, 0, 700], [3, 2, 4]), ([0, 100, 31], [90, 40, 1])])
def test_rows_that_are_there_already(prev, new, dtype):
    f = Fold(8, 2, 128, 16, prev, new, dtype, present=True).step().check()
    with kv.KvFoldPagedCache(1, 8, 2, 128, 16, f.n_pages, dtype) as other:  # and put there by append alone
        for rows in other.view(0):
            rows.fill_(math.nan)
        for s, (k, v) in enumerate(zip(f.k, f.v)):
            at = torch.arange(len(k))
            other.append(0, k.cuda(), v.cuda(), (f.tables[s, at // 16].long() * 16 + at % 16).cuda())
        for got, want in zip(other.view(0), (f.k_pages, f.v_pages)):
            assert torch.equal(got.cpu().nan_to_num(5), want.nan_to_num(5))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("prev,new,holes", [
    ([200, 60, 300], [1, 1, 1], [(0, 0), (0, 1), (2, 3), (1, 0)]), ([200, 60, 300], [3, 1, 4], [(0, 1), (1, 0), (2, 2), (2, 4)]),
    ([200, 0, 700], [70, 40, 33], [(0, 0), (0, 2), (1, 0), (2, 1), (2, 10)]), ([20], [1], [(0, 0), (0, 1)]), ([5], [50], [(0, 0)])])
def test_pages_that_are_none(prev, new, holes, page, dtype):
    """Keys of pages that the table does not name are seen by nobody, and a row that sees none has zeros and -inf."""
    counts = [-(-(p + n) // page) for p, n in zip(prev, new)]
    f = Fold(8, 2, 128, page, prev, new, dtype, holes=[(s, j) for s, j in holes if j < counts[s]])
    f.step().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prev,new", [([40, 3, 100], [4, 3, 2]), ([100, 7, 0], [40, 70, 64]), ([0, 64], [200, 129])])
def test_rows_do_not_take_harm_from_what_they_do_not_see(prev, new, dtype):
    """Each sequence's last rows of K and V are not finite: the rows before them see nothing of that."""
    f = Fold(8, 2, 128, 32, prev, new, dtype, seed=5)  # (the reference is of the rows as they were drawn)
    for s in range(len(new)):
        last = f.cu[s + 1] - 1
        for t in f.dev[1:]:
            t[last] = math.nan
            t[last, 0, :3] = torch.tensor([math.inf, -math.inf, 1.0]).to(t.dtype)
            if new[s] > 20:
                t[last - 5, 1, 7] = math.inf
    f.step().check(rows=[max(0, n - (6 if n > 20 else 1)) for n in new])


def test_a_long_sequence_beside_short_ones_and_many_pieces():
    f = Fold(8, 2, 128, 64, [30000, 1, 500, 0, 2300], [1] * 5).step().check().check_pages()
    again = Fold(8, 2, 128, 64, [30000, 1, 500, 0, 2300], [1] * 5).step()
    assert torch.equal(f.out, again.out) and torch.equal(f.lse, again.lse)
    for _ in range(3):  # the same workspace again, and the same bits
        out = f.out.clone()
        f.step()
        assert torch.equal(out, f.out)


def test_bounds_that_are_wide_and_layers():
    f = Fold(8, 2, 128, 32, [300, 7], [2, 1], layers=3, layer=2, max_new=4, max_len=5000).step().check().check_pages()
    for layer in (0, 1):
        for rows in f.cache.view(layer):
            rows.fill_(1.0)
    f.step().check().check_pages()
    assert all((rows == 1).all() for layer in (0, 1) for rows in f.cache.view(layer))


# ---- assign -----------------------------------------------------------------------------------------------------------------
def assigned(cache, page, lens, new, free, n_free, tables, n_slots, n_pages):
    dev = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    batch = kv.KvFoldBatch(cache, dev(tables) if len(tables) else torch.zeros((0, 3), dtype=torch.int32, device="cuda"), n_slots, 1, 1)
    for t in (batch.lens, batch.cu_new, batch.slots, batch.positions, batch.n_free, batch.status):
        t.fill_(99)
    cache.assign(batch, dev(lens), dev(new), dev(free), dev([n_free]))
    return [t.tolist() for t in (batch.tables, batch.lens, batch.cu_new, batch.slots, batch.positions)] + [batch.n_free.item(), batch.status.item()]


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("seqs,top,most", [(1, 40, 40), (7, 300, 5), (64, 2000, 1), (300, 50, 200), (1000, 100, 3), (3, 10, 9000)])
@pytest.mark.parametrize("change", [None, "pages", "table", "slots", "negative", "free"])
def test_assign(page, seqs, top, most, change):
    rng = np.random.default_rng(seqs + page)
    lens, new = rng.integers(0, top, seqs).tolist(), rng.integers(0, most + 1, seqs).tolist()
    if sum(new) == 0:
        new[0] = 1
    up = lambda n: -(-n // page)
    held, need = [up(p) for p in lens], [up(p + n) - up(p) for p, n in zip(lens, new)]
    n_pages = sum(held) + sum(need) + 4
    order = rng.permutation(n_pages).tolist()
    width = max(h + n for h, n in zip(held, need)) + 1
    tables, at = [], 0
    for h in held:
        tables.append(order[at:at + h] + [-1] * (width - h))
        at += h
    free = order[at:]
    n_free = len(free)
    free = free + [-1] * (n_pages - len(free))
    n_slots = sum(new) + 11
    if change == "pages":
        n_free = sum(need) - 1
    elif change == "table":
        width = max(h + n for h, n in zip(held, need)) - 1
        if width < 1:
            pytest.skip("no shorter table")
        tables = [r[:width] for r in tables]
    elif change == "slots":
        n_slots = sum(new) - 1
    elif change == "negative":
        lens[seqs // 2] = -5
    elif change == "free":
        n_free = n_pages + 1000  # (as many as there can be)
    with kv.KvFoldPagedCache(1, 1, 1, 64, page, n_pages) as cache:
        got = assigned(cache, page, lens, new, free, n_free, tables, n_slots, n_pages)
    want = R.assign(lens, new, free, n_free, tables, page, n_slots)
    for name, a, b in zip(("tables", "lens", "cu", "slots", "positions", "n_free", "status"), got, want):
        assert a == b, name


def test_assign_of_nothing():
    with kv.KvFoldPagedCache(1, 1, 1, 64, 16, 4) as cache:
        assert assigned(cache, 16, [], [], [3, 2, 1, 0], 4, [], 5, 4)[1:] == [[], [0], [-1] * 5, [-1] * 5, 4, 0]
        assert assigned(cache, 16, [3, 0], [0, 0], [3, 2, 1, 0], 4, [[1, 2], [3, 0]], 0, 4) == [[[1, 2], [3, 0]], [3, 0], [0, 0, 0], [], [], 4, 0]


# ---- the operators together ---------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_serving_loop_against_a_cache_for_each(dtype):
    """Prompts admitted, chunked and decoded, every tick's places from the lengths on the GPU: as if each sequence had a cache of its own."""
    hq, hkv, d, page, n_pages, seqs = 8, 2, 128, 32, 120, 5
    g = torch.Generator().manual_seed(3)
    cache = kv.KvFoldPagedCache(2, hq, hkv, d, page, n_pages, dtype)
    for layer in (0, 1):
        for rows in cache.view(layer):
            rows.fill_(math.nan)
    tables = torch.full((seqs, 40), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
    lens, n_free = torch.zeros(seqs, dtype=torch.int32, device="cuda"), torch.tensor([n_pages], dtype=torch.int32, device="cuda")
    own = [[kv.KvFoldCache(2, hq, hkv, d, 256, 1200, dtype)] for _ in range(seqs)]
    held = [0] * seqs
    for tick in ([70, 0, 33, 1, 250], [64, 100, 0, 40, 17], [1] * 5, [1, 1, 0, 1, 1], [3, 1, 4, 2, 1], [200, 1, 1, 1, 30], [1] * 5):
        n = sum(tick)
        held = [a + b for a, b in zip(held, tick)]
        batch = kv.KvFoldBatch(cache, tables, n + 2, max(tick), max(held))
        cache.assign(batch, lens, torch.tensor(tick, dtype=torch.int32).cuda(), free, n_free)
        lens, n_free = batch.lens, batch.n_free
        for layer in (0, 1):
            q, k, v = (draw(g, (n + 2, heads, d), dtype).cuda() for heads in (hq, hkv, hkv))
            out, lse = torch.full_like(q, 7), torch.full((hq, n + 2), 7.0, device="cuda")
            cache.step(layer, batch, q, k, v, out, lse=lse)
            at = 0
            for s, m in enumerate(tick):
                if m:
                    want, want_lse = torch.empty_like(q[at:at + m]), torch.empty((hq, m), device="cuda")
                    own[s][0].step(layer, q[at:at + m].contiguous(), k[at:at + m].contiguous(), v[at:at + m].contiguous(), want, lse=want_lse)
                    tol = 2e-2 if dtype == "bf16" else 1e-5  # each within its own of the definition (bf16: the steps' 2^-8 twice, of outputs of some units)
                    assert (out[at:at + m].double() - want.double()).abs().max() <= 2 * tol
                    assert (lse[:, at:at + m] - want_lse).abs().max() <= (3e-2 if dtype == "bf16" else 1e-4)  # (its queries are rounded once more)
                at += m
            assert (out[n:] == 7).all() and (lse[:, n:] == 7).all()
        assert batch.status.item() == 0 and lens.tolist() == held


def test_a_captured_tick_replayed():
    """assign, steps of two layers, lengths and free pages copied back: the graph runs on whatever they hold, its eager twin gives the same bits."""
    hq, hkv, d, page, n_pages, seqs = 8, 2, 128, 16, 64, 4

    def state():
        cache = kv.KvFoldPagedCache(2, hq, hkv, d, page, n_pages)
        for layer in (0, 1):
            for rows in cache.view(layer):
                rows.fill_(0.25)
        tables = torch.zeros((seqs, 20), dtype=torch.int32, device="cuda")
        x = dict(cache=cache, lens=torch.zeros(seqs, dtype=torch.int32, device="cuda"), n_free=torch.tensor([n_pages], dtype=torch.int32, device="cuda"),
                 free=torch.arange(n_pages, dtype=torch.int32, device="cuda"), new=torch.ones(seqs, dtype=torch.int32, device="cuda"),
                 batch=kv.KvFoldBatch(cache, tables, seqs, 1, 300), out=torch.zeros((2, seqs, hq, d), dtype=torch.bfloat16, device="cuda"),
                 lse=torch.zeros((2, hq, seqs), device="cuda"))
        x["qkv"] = torch.zeros((2, seqs, hq + 2 * hkv, d), dtype=torch.bfloat16, device="cuda")
        return x

    def tick(x):
        x["cache"].assign(x["batch"], x["lens"], x["new"], x["free"], x["n_free"])
        for layer in (0, 1):
            q, k, v = x["qkv"][layer].split((hq, hkv, hkv), 1)
            x["cache"].step(layer, x["batch"], q, k, v, x["out"][layer], lse=x["lse"][layer])
        x["lens"].copy_(x["batch"].lens)
        x["n_free"].copy_(x["batch"].n_free)

    a, b = state(), state()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        tick(a)  # (first use outside the capture)
    torch.cuda.current_stream().wait_stream(side)
    tick(b)
    with torch.cuda.graph(graph):
        tick(a)
    g = torch.Generator().manual_seed(8)
    for i in range(30):
        fresh = torch.randn((2, seqs, hq + 2 * hkv, d), generator=g).to(torch.bfloat16)
        new = torch.tensor([1, i % 2, 1, i % 3 == 0], dtype=torch.int32)
        for x in (a, b):
            x["qkv"].copy_(fresh)
            x["new"].copy_(new)
        graph.replay()
        tick(b)
        if i % 4 == 0:
            torch.cuda.synchronize()
        for name in ("out", "lse", "lens", "n_free"):
            assert torch.equal(a[name], b[name]), (i, name)
    assert a["lens"].tolist() == [31, 16, 31, 11]


def test_two_batches_on_two_streams():
    folds = [Fold(8, 2, 128, 16, [900 + i, 20, 300], [1, 1, 1], seed=i) for i in range(2)] + [Fold(8, 2, 128, 32, [100, 0], [200, 90 + i], seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in folds]
    torch.cuda.synchronize()
    for _ in range(5):
        for f, s in zip(folds, streams):
            with torch.cuda.stream(s):
                f.step()
    torch.cuda.synchronize()
    for f in folds:
        f.check().check_pages()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 3, 70])
def test_logits_that_jump(new, dtype):
    """Rising, falling and far: the reference follows."""
    for gain, shape in ((30.0, lambda j: 1.0 * (j > 500)), (60.0, lambda j: (j % 97 == 0) * 1.0), (0.2, lambda j: j * 1.0), (-90.0, lambda j: 1.0 * (j < 200))):
        f = Fold(4, 1, 64, 32, [900, 333], [new, new], dtype, seed=new)
        steer = torch.zeros(64)
        steer[0] = 8.0
        at = 0
        for s, n in enumerate(f.new):
            where = torch.arange(f.prev[s] + n)
            add = torch.tensor([gain * float(shape(int(j))) for j in where])
            k = f.k[s].float() * 0.1
            k[:, 0, 0] = add.clamp(-90, 90) if gain != 0.2 else add.clamp(-90, 180) / 2
            f.k[s] = k.to(R.TYPE[dtype])
            p = f.prev[s]
            f.k_pages[f.tables[s, where[:p] // 32].long(), :, where[:p] % 32] = f.k[s][:p]
            f.dev[1][at:at + n] = f.k[s][p:].cuda()
            f.q[at:at + n] = (f.q[at:at + n].float() * 0.1 + steer).to(R.TYPE[dtype])
            f.dev[0][at:at + n] = f.q[at:at + n].cuda()
            at += n
        f.cache.view(0)[0].copy_(f.k_pages)
        f.step().check()
