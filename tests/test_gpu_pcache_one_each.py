"""Steps of one token each, told by their places alone: a sequence without a place has no new token, as after an assignment that assigned nothing."""
import numpy as np
import pytest
import torch

import paper_2605_12471_amd as kv
import pcache_ref as R
from test_gpu_pcache import Fold, draw

pytestmark = pytest.mark.gpu
HEADS = [(8, 2, 128), (4, 1, 64), (18, 1, 64)]  # (the last on a prompt's kernels)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("prev", [[0, 5, 300, 64, 1], [9000, 40, 700, 3, 0]])
def test_sequences_without_a_place(hq, hkv, d, prev, dtype):
    f = Fold(hq, hkv, d, 32, prev, [1] * 5, dtype, one_each=True)
    for s, place in ((1, -1), (3, f.n_pages * 32)):
        f.batch.slots[s] = place
        f.slots[s] = f.slots[0]  # (stored twice in the expected pages: the row that lies there)
        f.kn[s], f.vn[s] = f.kn[0], f.vn[0]
    f.step().check(rows=[1, 0, 1, 0, 1]).check_pages()
    assert (f.out[[1, 3]] == 77).all() and (f.lse[:, [1, 3]] == 77).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("captured", [False, True])
def test_a_tick_that_runs_out_of_pages(captured, native, hq, hkv, d, dtype):
    """Nothing is assigned, and the step that follows changes nothing; with a page more both do their work."""
    page, seqs, n_pages = 16, 3, 8
    cache = kv.KvFoldPagedCache(1, hq, hkv, d, page, n_pages, dtype)
    if not native:
        cache._bound = None
    g = torch.Generator().manual_seed(4)
    for rows in cache.view(0):
        rows.copy_(draw(g, tuple(rows.shape), dtype))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    tables = i32([[0, 1, -1], [2, -1, -1], [3, -1, -1]])
    batch = kv.KvFoldBatch(cache, tables, seqs, 1, 48, one_each=True)
    q, k, v = (draw(g, (seqs, heads, d), dtype).cuda() for heads in (hq, hkv, hkv))
    out, lse = torch.zeros_like(q), torch.zeros((hq, seqs), device="cuda")
    lens, new, free, n_free = i32([20, 16, 5]), i32([1, 1, 1]), i32([4, 5, 6, 7, -1, -1, -1, -1]), i32([4])

    def tick():
        cache.assign(batch, lens, new, free, n_free)
        cache.step(0, batch, q, k, v, out, lse=lse)

    if captured:
        cache.step(0, kv.KvFoldBatch(cache, tables, seqs, 1, 48, one_each=True), q, k, v, out)  # (first use outside the capture: nobody has a place)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            tick()
    run = graph.replay if captured else tick
    for _ in range(3):
        n_free.fill_(0)  # the second request lacks a page
        before = [t.clone() for t in cache.view(0)]
        out.fill_(77), lse.fill_(77)
        run()
        torch.cuda.synchronize()
        assert batch.status.item() == 1 and batch.lens.tolist() == [20, 16, 5] and (out == 77).all() and (lse == 77).all()
        assert all(torch.equal(a, b) for a, b in zip(cache.view(0), before))
    n_free.fill_(4)
    run()
    assert batch.status.item() == 0 and batch.slots.tolist() == [20, 7 * 16, 3 * 16 + 5]
    for s, (p, numbers) in enumerate(((20, [0, 1]), (16, [2, 7]), (5, [3]))):
        rows = [t[numbers].transpose(1, 2).reshape(-1, hkv, d)[:p + 1].cpu() for t in cache.view(0)]
        assert all(torch.equal(r[p], x[s].cpu()) for r, x in zip(rows, (k, v)))
        ref, ref_lse, mean_abs, span = R.attend(q[s:s + 1].cpu(), *rows, np.ones((1, p + 1), dtype=bool), d ** -0.5)
        tol, tol_lse = R.bounds(ref, ref_lse, mean_abs, span, d, p + 1, dtype)
        assert (np.abs(out[s:s + 1].cpu().double().numpy() - ref) <= tol).all() and (np.abs(lse[:, s:s + 1].cpu().double().numpy() - ref_lse) <= tol_lse).all()
