"""Exact attention, and attention over the cache, of finite values of V of up to 2^127, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests.gpu_harness import DEV, tdtype
from tests.test_gpu_exact_attention import Problem
from tests.test_gpu_kv_cache import Serving

pytestmark = pytest.mark.gpu

# one row tile of 32, tiles of 128 (bf16), 129 to 256 features, shares of the keys (few, many)
PROMPTS = [([70, 33], [70, 200], 4, 2, 64), ([40, 90], [40, 90], 64, 64, 128), ([64, 20], [64, 150], 64, 64, 64), ([50], [64], 64, 64, 256), ([20], [300], 2, 1, 256),
           ([1], [3000], 4, 2, 64), ([2], [1030], 8, 1, 128), ([90, 50], [700, 520], 4, 2, 40), ([2], [1030], 8, 1, 256)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", range(len(PROMPTS)))
def test_large_values_of_a_prompt(shape, causal, dtype):
    p = Problem(*PROMPTS[shape], dtype, causal)
    t = tdtype(dtype)
    g = torch.Generator(device=DEV).manual_seed(shape)
    small = p.V
    # of any sign, and all of them alike, to where the sum of two is no float
    p.V = (2.0 ** 127 * (2 * torch.rand(p.V.shape, generator=g, device=DEV) - 1) * (1 - 2.0 ** -7)).to(t)
    p.call().check()
    p.V = torch.full_like(p.V, 1.6e38)
    p.call().check()
    # columns that are large beside ones that are not, odd values in rows that some do not see and in foreign ones
    p.V = small.clone()
    p.V[:, :, 3] = (p.V[:, :, 3].float().clamp(-4, 4) * 3e37).to(t)
    p.V[p.k_off[-1] - 3, 0, 3], p.V[p.k_off[-1] - 2, 0, 5], p.V[0], p.V[-1] = math.inf, -math.inf, math.nan, math.inf
    p.call().check()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [2, 64])
@pytest.mark.parametrize("value", [1e37, 2e36])
def test_equal_keys_and_keys_above_the_reference(value, heads, dtype):
    """64 equal keys of 1e37; and keys whose weight is a little below 2^8 of what came before them."""
    p = Problem([40], [64], heads, heads, 64, dtype, False)
    p.K.zero_()
    p.V.fill_(value)
    p.call().check()
    p = Problem([40], [700], heads, heads, 64, dtype, False)
    p.K.zero_()
    p.Q.zero_()
    p.Q[:, :, 0] = 8.0
    p.K[p.k_off[0] + 300:, :, 0] = 5.375                          # scores 0, then 5.375: a factor of 2^7.75
    p.V.fill_(1.0)
    p.V[p.k_off[0] + 300:] = value
    p.call().check()


CACHES = [(64, 128, 8, 2, [64, 65], [1, 1]), (16, 64, 3, 3, [200, 17], [1, 1]), (32, 80, 16, 1, [100, 129], [3, 1]), (128, 256, 4, 2, [300, 5], [1, 2]),
          (64, 128, 16, 2, [130, 40], [8, 5]), (64, 64, 4, 1, [5000, 100], [1, 1])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("case", range(len(CACHES)))
def test_large_values_of_the_cache(case, weights, dtype):
    page, d, Hq, Hkv, lens, rows = CACHES[case]
    for kind in ("any", "equal", "column"):
        s = Serving(len(lens), Hq, Hkv, d, page, -(-max(lens) // page) + 1, dtype, seed=case)
        n = sum(lens) + 3
        K, V = s.rows(n, Hkv), s.rows(n, Hkv)
        if kind == "any":
            V = (2.0 ** 126 * (2 * torch.rand(V.shape, device=DEV) - 1)).to(V.dtype)
        elif kind == "equal":
            V.fill_(1.6e38)
        else:
            V[:, :, 3] = (V[:, :, 3].float().clamp(-4, 4) * 3e37).to(V.dtype)
        s.store(lens, K, V)
        W = s.weights() if weights else None
        s.check_attention(s.reference(), *s.attend(rows, W=W), W=W, W_before=np.zeros(s.weights().shape))
