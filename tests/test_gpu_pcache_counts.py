"""Sequences with more new tokens than the batch says that any has: the first of them are what they would be, the others are left alone."""
import pytest
import torch

from test_gpu_pcache import Fold

pytestmark = pytest.mark.gpu


CASES = [
    (8, 2, 128, [20, 0, 300, 31], [10, 5, 4, 2], 4, None),            # decoding
    (8, 2, 128, [20, 0, 300, 31], [2, 2, 9, 1], 1, None),
    (3, 3, 64, [9000, 5], [17, 40], 16, None),
    (8, 2, 128, [20, 0, 300], [100, 33, 70], 33, None),               # short prompts and chunks
    (18, 1, 64, [5, 0], [3, 1], 1, None),
    (8, 2, 128, [700, 0, 64], [300, 265, 149], 150, 3000),            # long ones
    (4, 1, 64, [6000], [400], 65, 7000)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("present", [False, True])
@pytest.mark.parametrize("hq,hkv,d,prev,new,most,bound", CASES)
def test_more_new_tokens_than_any_has(hq, hkv, d, prev, new, most, bound, present, dtype):
    f = Fold(hq, hkv, d, 16, prev, new, dtype, max_new=most, max_len=bound, width=450 if bound else 0, pad=2, lead=1, present=present)
    counts = [min(n, most) for n in new]
    f.step().check(rows=counts)
    taken = torch.zeros(f.rows, dtype=torch.bool)
    for s, n in enumerate(counts):
        taken[f.cu[s]:f.cu[s] + n] = True
    assert (f.out.cpu()[~taken] == 77).all() and (f.lse.cpu()[:, ~taken] == 77).all()
