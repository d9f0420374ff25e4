"""Eviction of tokens whose codes are all zero, out of blocks of large scales: they stay zeros, with their signs, whatever scale
the destination gets."""
import pytest
import torch

from tests.gpu_harness import DEV
from tests.test_gpu_kv_cache import Serving, evict_and_check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,d", [(16, 16), (64, 128), (128, 256)])
@pytest.mark.parametrize("small", [None, -118, 3])
@pytest.mark.parametrize("exponent", [9, 10, 60, 120])
def test_zeros_of_blocks_with_large_scales(exponent, small, page, d):
    """Three source blocks a head.  The first and the last have the scale 2^exponent for one token that goes (its code times that
    scale is a float), the others' codes are 0 and -0; `small`: the scale's exponent of the block between them, all of it kept, else it is zeros too."""
    s = Serving(1, 2, 2, d, page, 4, "bf16", tables=2)
    s.lengths[0] += 3 * page
    t, n = s.tables[0][0].long(), 3 * page
    K, V = s.K.view(torch.uint8), s.V.view(torch.uint8)
    signs = (torch.arange(page * d, device=DEV) % 3 == 0).to(torch.uint8).mul(0x80).view(page, d)
    for j in range(3):
        if j == 1 and small is not None:
            s.Ks[t[j]], s.Vs[t[j]] = 2.0 ** small, 2.0 ** small
            continue
        s.Ks[t[j]], s.Vs[t[j]] = 2.0 ** exponent, 2.0 ** exponent
        K[t[j]], V[t[j]] = signs, signs.t()
        K[t[j], :, 5], V[t[j], :, :, 5] = 0x70, 0xf0             # 128, -128: the token that goes
    W = s.weights(1.0)
    W[:, :, 5], W[:, :, 2 * page + 5] = 0.0, 0.0
    if small is None:
        W[:, :, page + 5] = 0.0
    budget = n - (3 if small is None else 2)
    evict_and_check(s, W, budget, 0)
    # -0 stays -0
    order = [i for i in range(n) if W[0, 0, i] != 0]
    to = s.tables[1][0].long()
    for i, slot in enumerate(order):
        if small is not None and page <= slot < 2 * page:
            continue
        row = s.K.view(torch.uint8)[to[i // page], 0, i % page]
        col = s.V.view(torch.uint8)[to[i // page], 1, :, i % page]
        assert torch.equal(row, signs[slot % page]) and torch.equal(col, signs[slot % page]), (i, slot)


@pytest.mark.parametrize("least", [-118, -30])
def test_a_block_that_is_left_without_its_outlier(least):
    """One outlier of 3e5 among values of at most 1: stored, its neighbours' codes are zeros; evicted without it, they stay zeros."""
    s = Serving(1, 1, 1, 32, 16, 4, "f32", tables=2)
    K = s.rows(2 + 40 + 1, 1).clamp(-1, 1)
    K[2 + 7, 0, 3] = 3e5
    K[2 + 16:2 + 32] *= 2.0 ** least
    r = s.reference()
    s.store([40], K, K.flip(-1).contiguous(), reference=r)
    s.same_as(r)
    W = s.weights(1.0)
    W[:, :, 7] = 0.0
    evict_and_check(s, W, 39, 0)
    Q, O, lse, _ = s.attend([1], i=1)
    assert torch.isfinite(O).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("low,high", [(-118, -118), (120, 120), (-118, 120), (100, 112)])
def test_small_codes_at_the_ends_of_the_scales(low, high):
    """Subnormal codes, zeros and the largest whose value is a float, under the least and greatest scales there are."""
    s = Serving(1, 1, 1, 64, 32, 4, "bf16", tables=2)
    s.lengths[0] += 4 * 32
    t = s.tables[0][0].long()
    K, V = s.K.view(torch.uint8), s.V.view(torch.uint8)
    K[t], V[t] = torch.randint(0, 16, K[t].shape, device=DEV, dtype=torch.uint8), torch.randint(0, 16, V[t].shape, device=DEV, dtype=torch.uint8)
    for j, e in enumerate((low, high, high, low)):
        s.Ks[t[j]], s.Vs[t[j]] = 2.0 ** e, 2.0 ** e
    K[t[1], :, 20, 3], V[t[1], :, 4, 11] = 0x77, 0xf7            # 240: under 2^120 as large as a float goes
    K[t[2], :, 6, 60], V[t[2], :, 61, 9] = 0x7f, 0xff
    W = s.weights(1.0)
    W[:, :, ::7] = 0.0
    evict_and_check(s, W, int((W[0, 0] != 0).sum()), 0)
