"""The 8-bit cache's step where blocks of V are zero, tiny or as large as bf16 goes: what V is counts in the output alone, not in the softmax."""
import math

import numpy as np
import pytest
import torch

import paper_2605_12471_amd as kv
import qcache_ref as R
from test_gpu_qcache import Fold, draw

pytestmark = pytest.mark.gpu


def two_levels(n, hq, hkv, d, below):
    """q with one channel, and the two key rows whose logits under it are 0 and about -below; that logit as the cache holds it."""
    q = torch.zeros((n, hq, d))
    q[:, :, 0] = 16
    k = torch.zeros((2, hkv, d))
    k[1, :, 0] = -below * math.sqrt(d) / 16
    k = k.to(torch.bfloat16)
    scale = np.float32(abs(float(k[1, 0, 0]))) / np.float32(127)
    return q.to(torch.bfloat16), k[:1], k[1:], -16 * 127 * float(scale) / math.sqrt(d)


def sum_bound(steps, logit):
    """What a log-sum-exp may be off by where `steps` sums of blocks follow one another: each addition by 2^-24 of the sum, the 64 in a block and the
    meeting of wavefronts and pieces by 64 + 64 more, the weights by 2^-22 and the rounding of their exponents, 2^-24 of each three times;
    the logarithm and its own rounding by 2^-22 of the result's magnitude, at most 8 here."""
    return (steps + 128) * 2.0 ** -24 + 2.0 ** -22 + abs(logit) * 1.5 * 3 * 2.0 ** -24 + 8 * 2.0 ** -22


@pytest.mark.parametrize("value", [0.0, 2.0 ** -110])
@pytest.mark.parametrize("hq,hkv,d,prev,n", [(32, 8, 128, 129024, 2048), (40, 2, 64, 126976, 4096)])
def test_keys_without_values_count_in_the_sum(hq, hkv, d, prev, n, value):
    """Rows 64 ... of V are nothing, and their keys 27 octaves below the first: 130 thousand of them are 9e-4 of the softmax's sum."""
    q, first, rest, logit = two_levels(n, hq, hkv, d, 18.8)
    cache = kv.KvFoldQuantCache(1, hq, hkv, d, n, prev + n)
    ones, none = torch.ones((1, hkv, d), dtype=torch.bfloat16, device="cuda"), torch.full((1, hkv, d), value, dtype=torch.bfloat16, device="cuda")
    k0, k1 = first.cuda(), rest.cuda()
    cache.append(0, torch.cat((k0, k1.expand(63, hkv, d))), ones.repeat(64, 1, 1))
    cache.append(0, k1.expand(prev - 64, hkv, d), none.expand(prev - 64, hkv, d))
    out, lse = torch.empty((n, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((hq, n), device="cuda")
    cache.step(0, q.cuda(), k1.repeat(n, 1, 1), none.repeat(n, 1, 1), out, lse=lse)
    others = prev + np.arange(n)           # keys at the lower level that a row sees
    want = np.log1p(others * math.exp(logit))
    tol = sum_bound((prev + n) / 64, logit)
    assert 4 * tol < want.min()
    assert np.abs(lse.cpu().double().numpy() - want).max() <= tol
    mean = (1 + 63 * math.exp(logit)) / (1 + others * math.exp(logit))
    assert (np.abs(out.cpu().double().numpy() - mean[:, None, None]) <= 2.0 ** -8 * 2 * 1.01 * mean[:, None, None] + 2 * tol).all()


def test_keys_without_values_count_in_the_sum_of_a_decoding_step():
    """33 million of them, a level above them in four blocks of every piece, one for each of its wavefronts."""
    hq, hkv, d, pieces = 4, 1, 64, 24
    q, first, rest, logit = two_levels(1, hq, hkv, d, 18.8)
    per_piece = 64 * 21840
    cache = kv.KvFoldQuantCache(1, hq, hkv, d, 1, pieces * per_piece + 64)
    ones, none = (torch.full((1, hkv, d), x, dtype=torch.bfloat16, device="cuda") for x in (1.0, 0.0))
    k0, k1 = first.cuda(), rest.cuda()
    marked = torch.cat((k0, k1.expand(63, hkv, d))).repeat(4, 1, 1)
    for _ in range(pieces):
        cache.append(0, k1.expand(64 * 100, hkv, d), none.expand(64 * 100, hkv, d))
        cache.append(0, marked, ones.repeat(256, 1, 1))
        cache.append(0, k1.expand(per_piece - 64 * 104, hkv, d), none.expand(per_piece - 64 * 104, hkv, d))
    out, lse = torch.empty((1, hq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((hq, 1), device="cuda")
    cache.step(0, q.cuda(), k1, none, out, lse=lse)
    above, below = 4 * pieces, pieces * (per_piece - 4) + 1
    want, least = math.log(above + below * math.exp(logit)), math.log(above)
    tol = sum_bound(per_piece / 64 / 4 + 1, logit)
    assert 4 * tol < want - least
    assert np.abs(lse.cpu().double().numpy() - want).max() <= tol
    mean = (above + above * 63 * math.exp(logit)) / (above + below * math.exp(logit))
    assert np.abs(out.cpu().double().numpy() - mean).max() <= 2.0 ** -8 * 2 * 1.01 * mean + 2 * tol


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 5, 20, 300])
@pytest.mark.parametrize("gain", [0.0, 1e-36, 1e-28, 1e-6])
def test_steps_over_blocks_of_tiny_values(d, n, gain):
    """Every other run of blocks, or all of them, with tiny values, the last, incomplete one among them."""
    for every in (1, 2):
        f = Fold(8, 2, d, 1000 + n + 30, seed=n)
        _, k, v = f.chunk(1000)
        v[(torch.arange(1000) // 128) % every == 0] *= gain
        f.cache.append(0, k.cuda(), v.cuda())
        f.joined(k, v)
        q, k, v = f.chunk(n)
        f.step(n, data=(q, k, v * gain if every == 1 else v))
        f.step(1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 3, 20, 300])
@pytest.mark.parametrize("block", [0, 2, 5, 9, 14])
@pytest.mark.parametrize("rise", [0.0, 4.0, 7.0, 10.0, 25.0])
def test_an_infinity_among_the_values(d, n, block, rise):
    """A key's value is infinite, taken for the largest number, and its logit `rise` above the others'."""
    f = Fold(8, 2, d, 1030 + n, seed=block)
    q, k, v = f.chunk(1030)
    k[:, :, 0] = 0
    k[64 * block + 17, :, 0] = 4
    v[64 * block + 17, :, 3], v[64 * block + 17, 0, 5] = math.inf, -math.inf
    f.cache.append(0, k.cuda(), v.cuda())
    f.joined(k, v)
    q, k, v = f.chunk(n)
    q = q * 0.1
    q[:, :, 0], k[:, :, 0] = rise * math.sqrt(d) / 4, 0
    # (the row's mean has to be some way below the largest number, which the output may else be rounded up from)
    f.step(n, data=(q, k, v))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gain", [2.0 ** 30, 2.0 ** 60, 2.0 ** 76, 2.0 ** 80, 2.0 ** 84, 2.0 ** 88, 2.0 ** 118])
@pytest.mark.parametrize("profile", [lambda j: 20.0 * (j >= 700), lambda j: 30.0 * (j >= 500), lambda j: 38.0 * (j >= 1100), lambda j: 41.0 * (j >= 300), lambda j: 60.0 * (j >= 1100),
                                     lambda j: 0.4 * j])
def test_logits_that_jump_where_values_are_large(d, gain, profile):
    """Weights far above their row's reference, times values far above 1."""
    hq, hkv, prev, n = 16, 8, 1400, 1000
    f = Fold(hq, hkv, d, prev + n)
    g = torch.Generator().manual_seed(d)
    u = torch.nn.functional.normalize(torch.randn(d, generator=g), dim=0)
    level = torch.tensor([float(profile(j)) for j in range(prev + n)])
    k = (0.1 * torch.randn((prev + n, hkv, d), generator=g) + 0.5 * level[:, None, None] * u).to(torch.bfloat16)
    v = (gain * torch.randn((prev + n, hkv, d), generator=g)).to(torch.bfloat16)
    q = (0.1 * torch.randn((n, hq, d), generator=g) + 2 * math.sqrt(d) * u).to(torch.bfloat16)
    f.cache.append(0, k[:prev].cuda(), v[:prev].cuda())
    f.joined(k[:prev], v[:prev])
    f.step(n, data=(q, k[prev:], v[prev:]))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 5, 20, 300])
def test_steps_over_numbers_that_are_hard_to_hold(d, n):
    """Blocks of V that are zero, tiny, large, with one large element, or not finite, one behind the other."""
    f = Fold(4, 2, d, 64 * 12 + n + 2)
    q, k, v = f.chunk(64 * 12)
    v[64:128] = 0
    v[128:192] *= 1e-36
    v[192:256] *= 2.0 ** 100
    v[256:320, 0, 0] = 1000
    v[320, 0, 1], v[321, 0, 1], v[322, 0, 1] = math.inf, -math.inf, math.nan
    v[450:460] *= 2.0 ** 60
    f.cache.append(0, k.cuda(), v.cuda())
    f.joined(k, v)
    f.step(n)
    f.step(1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 3, 20, 40])
@pytest.mark.parametrize("prev", [30, 640 + 22, 64 * 40 + 10])
def test_infinities_in_the_last_block(d, n, prev):
    """Rows that are not a whole block are held as they came: several of the largest numbers, of either sign, with like weights."""
    f = Fold(8, 2, d, prev + n + 1, seed=prev)
    _, k, v = f.chunk(prev)
    first = prev // 64 * 64
    v[first + 2:first + 9, :, 3], v[first + 5, 0, 4], v[first + 6, 0, 4], v[first + 7, 1, 5] = math.inf, math.inf, -math.inf, math.nan
    k[first:, :, 0] = 6.0
    f.cache.append(0, k.cuda(), v.cuda())
    f.joined(k, v)
    q, k, v = f.chunk(n)
    q[:, :, 0] = 6.0
    f.step(n, data=(q * 0.5, k, v))
    f.step(1)
