"""Keys whose logits are -inf, where a row's reference is found: they have no weight, the others theirs."""
import math

import pytest
import torch

import pcache_ref as R
from test_gpu_pcache import Fold

pytestmark = pytest.mark.gpu


def hide(f, pages, shift):
    """Keys of these pages (of every sequence) are -inf in a column in which all queries are positive; all other logits lie near `shift`."""
    d, col = f.d, 3
    of = R.TYPE[f.dtype]
    f.q[:, :, col] = f.q[:, :, col].abs() + 0.1
    f.q[:, :, 0] = 16.0
    for s, n in enumerate(f.new):
        p, at = f.prev[s], f.cu[s]
        where = torch.arange(p + n)
        k = f.k[s]
        k[:, :, 0] = shift * math.sqrt(d) / 16.0
        k[:, :, col] = 0.0
        mine = [j for j in pages if j * f.page < p]
        gone = torch.zeros(p + n, dtype=torch.bool)
        for j in mine:
            gone[j * f.page:min((j + 1) * f.page, p)] = True
        k[gone, :, col] = -math.inf
        f.k[s] = k.to(of)
        f.k_pages[f.tables[s, where[:p] // f.page].long(), :, where[:p] % f.page] = f.k[s][:p]
        f.kn[at:at + n] = f.k[s][p:]
        visible = f.visible(s) & ~gone.numpy()[None, :]
        f.seen = getattr(f, "seen", {})
        f.seen[s] = visible
    f.visible = lambda s: f.seen[s]
    f.dev[0].copy_(f.q.cuda())
    f.dev[1].copy_(f.kn.cuda())
    f.cache.view(f.layer)[0].copy_(f.k_pages)


@pytest.mark.parametrize("shift", [0.0, -140.0, 60.0])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 1, 64)])
@pytest.mark.parametrize("dtype,bound", [("bf16", 8000), ("bf16", None), ("f32", None)])
@pytest.mark.parametrize("prev,new,pages", [([700, 333], [140, 150], [0]), ([700, 96], [140, 150], [0, 1, 2, 4, 7]), ([6000], [200], [0] + list(range(8, 180, 2))),
                                            ([6000], [200], range(187)), ([300, 40], [1, 1], [0]), ([3000, 64], [3, 2], range(0, 80, 3)), ([128], [40], [0, 1, 2, 3])])
def test_the_first_keys_have_no_weight(prev, new, pages, dtype, bound, hq, hkv, d, shift):
    f = Fold(hq, hkv, d, 32, prev, new, dtype, seed=3, max_len=bound, width=260 if bound else 0)
    hide(f, pages, shift)
    f.step().check().check_pages()
