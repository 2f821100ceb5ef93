"""Calls of the cache in pages: what is refused, before anything is enqueued, and the native form of the binding beside the plain one."""
import ctypes

import pytest
import torch

import paper_2605_12471_amd as kv
from paper_2605_12471_amd import binding
from test_gpu_pcache import Fold

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE, PAGES, SEQS, N = 8, 2, 128, 16, 40, 3, 6


class Call:
    """Arguments of one good step on the C entry, to be changed one at a time."""

    def __init__(self, new=2):
        dev = "cuda"
        self.cache = kv.KvFoldPagedCache(2, HQ, HKV, D, PAGE, PAGES)
        for layer in (0, 1):
            for rows in self.cache.view(layer):
                rows.fill_(0.5)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
        self.tables = torch.arange(SEQS * 4, dtype=torch.int32, device=dev).reshape(SEQS, 4)
        self.lens, self.cu = i32([10, 20, 30]), i32([0, 2, 4, 6])
        self.slots = torch.tensor([8, 9, 82, 83, 156, 157], device=dev)
        self.q, self.k, self.v = (torch.ones((N, heads, D), dtype=torch.bfloat16, device=dev) for heads in (HQ, HKV, HKV))
        self.out, self.lse = torch.full_like(self.q, 3), torch.full((HQ, N), 3.0, device=dev)
        self.batch = binding.make_batch(SEQS, N, new, 64, self.tables.data_ptr(), 4, self.lens.data_ptr(), self.cu.data_ptr(), self.slots.data_ptr())
        need = kv.kvfold_pcache_workspace_bytes(self.cache.handle, self.batch)
        self.space = torch.zeros(need, dtype=torch.uint8, device=dev)
        self.layer = 0
        self.at = dict(q=self.q.data_ptr(), k=self.k.data_ptr(), v=self.v.data_ptr(), out=self.out.data_ptr(), lse=self.lse.data_ptr(), space=self.space.data_ptr(), bytes=need)

    def __call__(self, **change):
        a, b = dict(self.at), binding.kvfold_batch_t.from_buffer_copy(self.batch)
        layer = change.pop("layer", 0)
        for name, value in change.items():
            if name in a:
                a[name] = value
            else:
                setattr(b, name, value)
        return kv.load_library().kvfold_pcache_step(self.cache.handle, layer, ctypes.byref(b), a["q"], a["k"], a["v"], a["out"], a["lse"], a["space"], a["bytes"],
                                                    torch.cuda.current_stream().cuda_stream)

    def untouched(self):
        torch.cuda.synchronize()
        return bool((self.out == 3).all() and (self.lse == 3).all() and (self.space == 0).all() and all((rows == 0.5).all() for i in (0, 1) for rows in self.cache.view(i)))


@pytest.mark.parametrize("new", [2, 6])  # decoding, and a prompt's kernels
def test_steps_that_are_refused(new):
    c = Call(new)
    store = c.cache.view(0)[0].data_ptr()
    bad = [(dict(layer=-1), -2), (dict(layer=2), -2), (dict(q=None), -1), (dict(out=None), -1), (dict(space=None), -1), (dict(k=None), -1), (dict(v=None), -1),
           (dict(slots=None), -1), (dict(slots=None, k=None), -1), (dict(tables=None), -1), (dict(lens=None), -1), (dict(cu_new=None), -1), (dict(struct_size=3), -1),
           (dict(max_new=0), -1), (dict(n_tokens=-1), -1), (dict(n_seqs=-1), -1), (dict(q_stride=1), -1), (dict(q_stride=HQ * D - 8), -1), (dict(kv_stride=HKV * D - 8), -1),
           (dict(max_len=(1 << 30) + 1), -5), (dict(n_seqs=(1 << 20) + 1), -5), (dict(bytes=c.at["bytes"] - 1), -6), (dict(bytes=0), -6)]
    bad += [(dict([(name, c.at[name] + 8)]), -1) for name in ("q", "k", "v", "out")] + [(dict(space=c.at["space"] + 128), -1), (dict(lse=c.at["lse"] + 2), -1)]
    bad += [(dict([(name, getattr(c.batch, name) + 2)]), -1) for name in ("tables", "lens", "cu_new", "slots")]
    for x in ("out", "lse", "space"):  # what is written beside everything else
        bad += [(dict([(x, c.at[y])]), -1) for y in ("q", "k", "v", "out", "lse", "space") if y != x and c.at[y] % 256 == 0]
        bad += [(dict([(x, at)]), -1) for at in (store, c.cache.view(1)[1].data_ptr(), c.batch.slots, c.batch.tables, c.batch.lens, c.batch.cu_new)]
        bad += [(dict([(x, c.at[x]), ("q", c.at[x] + (0 if x != "out" else 16))]), -1)]
    bad += [(dict([(y, store)]), -1) for y in ("q", "k", "v", "slots", "tables", "lens", "cu_new")]
    for change, status in bad:
        assert c(**change) == status, change
    assert c.untouched()
    assert c() == 0 and c(lse=None) == 0 and c(k=None, v=None, slots=None) == 0 and c(n_tokens=0) == 0 and c(n_seqs=0) == 0
    torch.cuda.synchronize()
    assert not c.untouched()
    assert kv.kvfold_pcache_workspace_bytes(c.cache.handle, binding.make_batch(1, 1, 0, 1)) == 0


def test_appends_that_are_refused():
    c = Call()
    lib, h, stream = kv.load_library(), c.cache.handle, torch.cuda.current_stream().cuda_stream
    k, v, slots, store = c.at["k"], c.at["v"], c.slots.data_ptr(), c.cache.view(0)[0].data_ptr()
    for a, status in (((-1, k, v, 0, slots, 2), -2), ((2, k, v, 0, slots, 2), -2), ((0, None, v, 0, slots, 2), -1), ((0, k, None, 0, slots, 2), -1), ((0, k, v, 0, None, 2), -1),
                      ((0, k, v, 0, slots, -1), -1), ((0, k, v, 8, slots, 2), -1), ((0, k, v, HKV * D + 4, slots, 2), -1), ((0, k, v, -8, slots, 2), -1), ((0, k + 8, v, 0, slots, 2), -1),
                      ((0, k, v, 0, slots + 4, 2), -1), ((0, store, v, 0, slots, 2), -1), ((0, k, store, 0, slots, 2), -1), ((0, k, v, 0, store, 2), -1),
                      ((0, k, v, (1 << 31) + 8, slots, 2), -5)):
        assert lib.kvfold_pcache_append(h, *a, stream) == status, a
    assert c.untouched()
    assert lib.kvfold_pcache_append(h, 0, None, None, 0, None, 0, stream) == 0
    # places that are none are passed over; a stride may be any multiple of 16 bytes
    c.cache.append(0, c.k, c.v, torch.tensor([-1, PAGES * PAGE, 1 << 62, -(1 << 63), 3, (1 << 31) + 3], device="cuda"))
    wide = torch.full((2, HKV + 1, D), 7.0, dtype=torch.bfloat16, device="cuda")
    c.cache.append(0, wide[:, :HKV], wide[:, :HKV], torch.tensor([17, 18], device="cuda"))
    for rows in c.cache.view(0):
        want = torch.full_like(rows, 0.5)
        want[0, :, 3], want[1, :, 1:3] = 1, 7
        assert torch.equal(rows, want)


def test_assignments_that_are_refused():
    c = Call()
    lib, stream = kv.load_library(), torch.cuda.current_stream().cuda_stream
    i32 = lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    t = [c.lens, i32(3), i32(PAGES), i32(1), c.tables, i32(3), i32(4), torch.zeros(N, dtype=torch.int64, device="cuda"), i32(N), i32(1), i32(1)]
    lens, new, free, n_free, tables, after, cu, slots, positions, left, status = (x.data_ptr() for x in t)
    good = [SEQS, lens, new, free, n_free, tables, 4, after, cu, slots, positions, N, left, status]
    call = lambda *changes: lib.kvfold_pcache_assign(c.cache.handle, *[dict(changes).get(i, x) for i, x in enumerate(good)], stream)
    assert call() == 0
    torch.cuda.synchronize()
    before = [x.clone() for x in t]
    for i in (1, 2, 3, 4, 5, 7, 8, 9, 12, 13):
        assert call((i, None)) == -1, i
        assert call((i, good[i] + 2)) == -1, i
    assert call((10, good[10] + 2)) == -1 and call((0, -1)) == -1 and call((11, -1)) == -1 and call((6, 0)) == -1
    assert call((0, (1 << 20) + 1)) == -5 and call((11, 1 << 31)) == -5 and call((6, 1 << 31)) == -5
    results = (5, 7, 8, 9, 10, 12, 13)
    for i in results:
        for j in (1, 2, 3, 4) + results:
            if i != j and (i != 9 or good[j] % 8 == 0):
                assert call((i, good[j])) == -1, (i, j)
        assert call((i, c.cache.view(1)[0].data_ptr())) == -1
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(t, before)) and c.untouched()
    assert call((10, None)) == 0  # no positions


@pytest.mark.parametrize("native", [True, False])
def test_what_the_binding_refuses(native):
    f = Fold(HQ, HKV, D, PAGE, [20, 3], [2, 1])
    if native:
        f.step()
        assert f.cache._bound is not None
    else:
        f.cache._bound = None
    q, k, v = f.dev
    out, lse = torch.zeros_like(q), torch.zeros((HQ, 3), device="cuda")
    good = dict(q=q, k_new=k, v_new=v, out=out, lse=lse)
    wide = torch.zeros((3, HKV, 2 * D), dtype=torch.bfloat16, device="cuda")
    for name, t in (("q", q.float()), ("q", q[:2]), ("q", q.cpu()), ("q", q[:, :4]), ("q", q.reshape(3, -1)), ("q", q.transpose(0, 1).contiguous().transpose(0, 1)),
                    ("q", q[:1].expand(3, -1, -1)), ("k_new", k[:, :1]), ("k_new", wide[:, :, :D]), ("k_new", wide[:, :, ::2]), ("v_new", v.half()), ("v_new", v.cpu()),
                    ("k_new", None), ("v_new", None), ("out", torch.zeros((3, HQ, 2 * D), dtype=torch.bfloat16, device="cuda")[..., :D]), ("out", out[:2]), ("out", out.float()),
                    ("lse", lse.double()), ("lse", lse.T), ("lse", lse[:, :2]), ("v_new", torch.zeros((3, HKV + 1, D), dtype=torch.bfloat16, device="cuda")[:, :HKV])):
        with pytest.raises(ValueError):
            f.cache.step(0, f.batch, **{**good, name: t})
    with pytest.raises(kv.KvFoldError):
        f.cache.step(1, f.batch, **good)
    for name, t in (("workspace", f.batch.workspace[:256].contiguous()), ):
        kept, f.batch.workspace = f.batch.workspace, t
        if t.numel() < kept.numel():
            with pytest.raises(kv.KvFoldError):
                f.cache.step(0, f.batch, **good)
        f.batch.workspace = kept
    for name in ("lens", "cu_new", "slots", "tables"):
        kept = getattr(f.batch, name)
        for t in (kept.cpu(), kept.float(), kept[:-1]):
            if name == "tables" and t.dtype == torch.int32 and t.is_cuda:
                continue
            setattr(f.batch, name, t)
            with pytest.raises(ValueError):
                f.cache.step(0, f.batch, **good)
        setattr(f.batch, name, kept)
    with pytest.raises(ValueError):
        f.cache.append(0, k, wide[:, :, :D], f.slots[:3].cuda())
    with pytest.raises(ValueError):
        f.cache.append(0, k, v, f.slots[:2].cuda())
    batch, i32 = f.batch, lambda n: torch.zeros(n, dtype=torch.int32, device="cuda")
    for a in ((i32(3), i32(2), i32(f.n_pages), i32(1)), (i32(2), i32(2).long(), i32(f.n_pages), i32(1)), (i32(2), i32(2), i32(f.n_pages - 1), i32(1)),
              (i32(2), i32(2), i32(f.n_pages), i32(2)), (i32(2).cpu(), i32(2), i32(f.n_pages), i32(1))):
        with pytest.raises(ValueError):
            f.cache.assign(batch, *a)
    with pytest.raises(kv.KvFoldError):  # lens after beside lens
        f.cache.assign(batch, batch.lens, i32(2), i32(f.n_pages), i32(1))
    for a in ((-1, 1, 1), (1 << 31, 1, 1), (3, 0, 1), (3, 1, 0), (3, 1 << 31, 1), (3, 1, (1 << 30) + 1)):
        with pytest.raises(ValueError):
            kv.KvFoldBatch(f.cache, f.batch.tables, *a)
    with pytest.raises(ValueError):
        kv.KvFoldBatch(f.cache, f.batch.tables.long(), 3, 1, 9)
    with pytest.raises(ValueError):
        kv.KvFoldBatch(f.cache, f.batch.tables[0], 3, 1, 9)
    with pytest.raises(ValueError):
        kv.KvFoldBatch(f.cache, f.batch.tables[:, :0], 3, 1, 9)
    with pytest.raises(ValueError):
        kv.KvFoldBatch(f.cache, f.batch.tables.T, 3, 1, 9)
    f.step().check().check_pages()
    f.cache.close()
    for _ in range(2):
        with pytest.raises(kv.KvFoldError):
            f.cache.step(0, f.batch, **good)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kw", [dict(prev=[20, 300], new=[1, 1], one_each=True), dict(prev=[20, 300], new=[2, 1], pad=2), dict(prev=[0, 300], new=[70, 40], fused=True),
                                dict(prev=[5, 3], new=[3, 4], present=True)])
def test_native_and_plain_are_the_same(kw, dtype):
    a, b = (Fold(HQ, HKV, D, PAGE, dtype=dtype, **kw) for _ in range(2))
    b.cache._bound = None
    stream = torch.cuda.Stream()
    for s in (None, stream.cuda_stream):
        for f in (a, b):
            f.step()
            if s:
                f.out.fill_(77), f.lse.fill_(77)
                torch.cuda.synchronize()
                k, v = (None, None) if f.present else f.dev[1:]
                f.cache.step(0, f.batch, f.dev[0], k, v, f.out, lse=f.lse, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(a.out, b.out) and torch.equal(a.lse, b.lse)
        a.check()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    got = []
    for f in (a, b):
        f.cache.assign(f.batch, i32([0, 5]), i32([1, 1]), torch.arange(f.n_pages, dtype=torch.int32, device="cuda"), i32([2]))
        got.append([t.tolist() for t in (f.batch.lens, f.batch.slots, f.batch.cu_new, f.batch.n_free, f.batch.status)])
    assert got[0] == got[1]


def test_storage_of_the_callers_and_views_that_stay():
    cfg = binding.make_pconfig(1, HQ, HKV, D, PAGE, 4, kv.KVFOLD_BF16)
    need = kv.kvfold_pcache_bytes_required(cfg)
    store = torch.zeros(need + 512, dtype=torch.uint8, device="cuda")
    at = (store.data_ptr() + 255) // 256 * 256
    cfg.kv_buffer, cfg.kv_buffer_bytes = at, need
    rc, h = kv.kvfold_pcache_create(cfg)
    assert rc == 0 and kv.kvfold_pcache_view(h, 0) == (0, at, at + need // 2)
    k = torch.ones((1, HKV, D), dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([PAGE + 2], device="cuda")
    assert kv.load_library().kvfold_pcache_append(h, 0, k.data_ptr(), k.data_ptr(), 0, slots.data_ptr(), 1, torch.cuda.current_stream().cuda_stream) == 0
    assert kv.kvfold_pcache_view(h, 1)[0] == -2 and kv.kvfold_pcache_destroy(h) == 0
    rows = store[at - store.data_ptr():][:need].view(torch.bfloat16).view(2, 4, HKV, PAGE, D)
    want = torch.zeros_like(rows)
    want[:, 1, :, 2] = 1
    assert torch.equal(rows, want)
    cache = kv.KvFoldPagedCache(1, HQ, HKV, D, PAGE, 4)
    view = cache.view(0)[1]
    view.fill_(2)
    del cache  # (the view keeps it)
    assert (view == 2).all()


def test_the_softmax_scale_is_the_callers():
    for scale, dtype in ((0.5, "bf16"), (0.01, "f32")):
        for prev, new in (([50], [1]), ([50, 0], [60, 40])):
            f = Fold(4, 1, 64, PAGE, prev, new, dtype)
            scaled = kv.KvFoldPagedCache(1, 4, 1, 64, PAGE, f.n_pages, dtype, softmax_scale=scale * 0.125)
            for a, b in zip(scaled.view(0), f.cache.view(0)):
                a.copy_(b)
            f.step()
            q = f.dev[0].float() / scale
            f2_out, f2_lse = torch.empty_like(f.out), torch.empty_like(f.lse)
            scaled.step(0, f.batch, q.to(f.dev[0].dtype), f.dev[1], f.dev[2], f2_out, lse=f2_lse)
            tol = 0 if scale == 0.5 else 1e-4  # (a factor of two changes no bits; else one rounding more of q: some 2^-24 of a logit's terms, which sum to some tens)
            assert (f2_out.float() - f.out.float()).abs().max() <= tol and (f2_lse - f.lse).abs().max() <= tol
