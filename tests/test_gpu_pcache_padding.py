"""Rows that belong to no sequence are not stored, whatever place they are given, in any kind of step."""
import math

import pytest
import torch

from test_gpu_pcache import Fold
from test_gpu_pcache_counts import CASES

pytestmark = pytest.mark.gpu
KINDS = [([40, 0, 70], [1, 2, 1], None), ([40, 0, 70], [30, 0, 41], None), ([5000], [40], None), ([700, 30], [140, 150], 2000)]  # decoding, short, in pieces, long


def unused(f, n):
    """Places in pages that no table names."""
    known = set(f.tables.flatten().tolist())
    page = next(p for p in range(f.n_pages) if p not in known)
    return page * f.page + torch.arange(n) % f.page


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 1, 64)])
@pytest.mark.parametrize("prev,new,bound", KINDS)
def test_places_of_rows_in_front_and_behind(prev, new, bound, hq, hkv, d, dtype):
    f = Fold(hq, hkv, d, 16, prev, new, dtype, lead=5, pad=7, max_len=bound, width=130)
    slots = f.slots.clone()
    slots[:5], slots[f.n_tokens:] = unused(f, 5), unused(f, 7)
    f.batch.slots.copy_(slots)
    f.step().check().check_pages()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("seqs,hq,hkv,d", [(63, 2, 2, 64), (64, 8, 8, 128), (65, 1, 1, 64), (257, 8, 2, 128), (1030, 2, 2, 64), (4200, 1, 1, 64)])
def test_empty_sequences_at_the_ends_and_between(seqs, hq, hkv, d, dtype):
    """One to eight tokens a wavefront of the rows' way to their places; sequences by the dozen, and thousands."""
    new = [0 if s % 3 == 0 or s < 5 or s > seqs - 9 else 17 + s % 4 if s % 5 else 1 for s in range(seqs)]
    f = Fold(hq, hkv, d, 16, [s % 37 for s in range(seqs)], new, dtype, lead=2, pad=9)
    slots = f.slots.clone()
    slots[:2], slots[f.n_tokens:] = unused(f, 2), unused(f, 9)
    f.batch.slots.copy_(slots)
    f.step().check().check_pages()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [4, 40])
def test_tokens_in_front_of_a_sequences_first_position(new, dtype):
    """A length below the number of new tokens: those that would lie in front of the first position see nothing and are not stored."""
    f = Fold(8, 2, 128, 16, [50, 0, 33], [new] * 3, dtype, pad=1)
    lens = [50 + new, new - 3, 33 + new]
    f.batch.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    slots = f.slots.clone()
    slots[f.cu[1]:f.cu[1] + 3] = unused(f, 3)
    slots[f.cu[1] + 3:f.cu[2]] = f.slots[f.cu[1]:f.cu[2] - 3]
    f.batch.slots.copy_(slots)
    f.step()
    f.check(rows=[new, 0, new])
    first = slice(f.cu[1], f.cu[1] + 3)
    assert (f.out[first] == 0).all() and (f.lse[:, first] == -math.inf).all()
    kept = torch.ones(f.rows, dtype=torch.bool)
    kept[first], kept[f.n_tokens:] = False, False
    view = torch.int16 if dtype == "bf16" else torch.int32
    for got, want, rows in zip(f.cache.view(0), (f.k_pages, f.v_pages), (f.kn, f.vn)):
        want = want.clone()
        want[slots[kept] // 16, :, slots[kept] % 16] = rows[kept]
        assert torch.equal(got.cpu().view(view), want.view(view))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,prev,new,most,bound", CASES)
def test_tokens_beyond_the_most_that_any_has(hq, hkv, d, prev, new, most, bound, dtype):
    f = Fold(hq, hkv, d, 16, prev, new, dtype, max_new=most, max_len=bound, width=450 if bound else 0, pad=2, lead=1).step()
    taken = torch.cat([torch.arange(f.cu[s], f.cu[s] + min(n, most)) for s, n in enumerate(new)])
    slots = f.slots[taken]
    view = torch.int16 if dtype == "bf16" else torch.int32
    for got, want, rows in zip(f.cache.view(0), (f.k_pages, f.v_pages), (f.kn, f.vn)):
        want = want.clone()
        want[slots // 16, :, slots % 16] = rows[taken]
        assert torch.equal(got.cpu().view(view), want.view(view))
