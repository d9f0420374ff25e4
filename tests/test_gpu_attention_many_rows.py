"""Exact attention and attention over the cache with more rows than one grid takes: as many as csat.h allows are computed."""
import numpy as np
import pytest
import torch

import paper_2507_02957_amd as csat
from tests.exact_reference import half_step
from tests.gpu_harness import DEV, tdtype
from tests.test_gpu_exact_attention import dev_ints
from tests.test_gpu_kv_cache import Serving

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,Hq,Hkv,n", [("f32", 16, 1, 131_100), ("bf16", 64, 1, 131_100), ("f32", 32, 2, 131_099)])
@pytest.mark.parametrize("causal", [False, True])
def test_prompt_of_more_than_65535_row_tiles(causal, dtype, Hq, Hkv, n):
    """The rows of one sequence against those of the same sequence in parts."""
    d, keys = 8, 40
    g = torch.Generator(device=DEV).manual_seed(1)
    Q, K, V = (torch.randn(m, h, d, generator=g, device=DEV).to(tdtype(dtype)) for m, h in ((n, Hq), (keys, Hkv), (keys, Hkv)))

    def call(first, count, seen):
        q, O, lse = Q[first:first + count], torch.full((count, Hq, d), 7.0, dtype=Q.dtype, device=DEV), torch.full((Hq, count), 7.0, device=DEV)
        dims = csat.make_packed_dims(1, Hq, Hkv, d, count, keys, count, keys, dtype, causal)
        ws = torch.empty(csat.csat_prompt_workspace_bytes(dims), dtype=torch.uint8, device=DEV)
        csat.csat_prompt_attention(dims, q, K, V, dev_ints([0, count]), dev_ints([0, seen]), 0.5, O, lse, ws)
        torch.cuda.synchronize()
        return O, lse
    O, lse = call(0, n, keys)
    # causal: only the last rows see keys, and each part's last rows those that they see of the whole
    cut = n - 20 if causal else n // 2
    # (another number of tiles may mean another kernel: what both may be off, the bounds of exact_reference.attend at the largest values)
    q, k, v = (float(x.float().abs().max()) for x in (Q, K, V))
    ds = 2.0 ** -24 * (d + 8) * 0.5 * d * q * k
    w = 2 * ds + 2.0 ** -24 * (keys + 32)
    bound = 2 * v * (w + half_step(dtype) * (2 if dtype == "bf16" else 1))
    for first, count, seen in ((0, cut, keys - (n - cut) if causal else keys), (cut, n - cut, keys)):
        o, l = call(first, count, seen)
        assert ((O[first:first + count].float() - o.float()).abs() <= bound).all()
        seen_rows = torch.isfinite(l)
        assert torch.equal(torch.isfinite(lse[:, first:first + count]), seen_rows)
        assert ((lse[:, first:first + count] - l)[seen_rows].abs() <= 2 * (w + 2.0 ** -23 * d * q * k)).all()
    assert causal == bool((lse == -float("inf")).any())


@pytest.mark.parametrize("max_pages", [1, 16])
def test_cache_attention_of_many_rows(max_pages):
    """131 100 rows of 32 heads, without and with shares of the keys, against the two halves of them."""
    n, Hq = 131_100, 32
    s = Serving(1, Hq, 1, 16, 64, max_pages, "bf16")
    s.lengths[0] += 50 if max_pages == 1 else 1000
    Q = s.rows(n, Hq)

    def call(q):
        O, lse = torch.full_like(q, 7.0), torch.full((Hq, q.shape[0]), 7.0, device=DEV)
        dims, cache = s.dims(q.shape[0], 1, q.shape[0], 1, causal=False), s.cache()
        ws = torch.empty(csat.csat_cache_workspace_bytes_without_weights(dims, cache), dtype=torch.uint8, device=DEV)
        csat.csat_cache_attention(dims, cache, q, dev_ints([0, q.shape[0]]), s.scale, 0.0, O, lse, None, ws)
        torch.cuda.synchronize()
        return O, lse
    O, lse = call(Q)
    parts = [call(q) for q in (Q[:n // 2], Q[n // 2:])]
    assert torch.equal(O, torch.cat([o for o, _ in parts])) and torch.equal(lse, torch.cat([l for _, l in parts], 1))
    assert torch.isfinite(O.float()).all() and (O != 7.0).any()


@pytest.mark.parametrize("max_pages", [1, 16])
def test_cache_attention_of_more_row_tiles_than_a_grid(max_pages):
    """67 million rows, the same query in all of them (a stride of 0), with a length of keys that takes one share and two."""
    n, Hq, d = 1_048_600, 64, 16
    s = Serving(1, Hq, 1, d, 64, max_pages, "f32")
    s.lengths[0] += 50 if max_pages == 1 else 1000
    Q = s.rows(1, 1).expand(n, Hq, d)
    O = torch.full((n, Hq, d), 7.0, device=DEV)
    dims, cache = s.dims(n, 1, n, 1, causal=False, Q=Q, O=O), s.cache()
    ws = torch.empty(csat.csat_cache_workspace_bytes_without_weights(dims, cache), dtype=torch.uint8, device=DEV)
    csat.csat_cache_attention(dims, cache, Q, dev_ints([0, n]), s.scale, 0.0, O, None, None, ws)
    torch.cuda.synchronize()
    one = torch.full((1, Hq, d), 7.0, device=DEV)
    dims = s.dims(1, 1, 1, 1, causal=False, Q=Q[:1], O=one)
    ws = torch.empty(csat.csat_cache_workspace_bytes_without_weights(dims, cache), dtype=torch.uint8, device=DEV)
    csat.csat_cache_attention(dims, cache, Q[:1], dev_ints([0, 1]), s.scale, 0.0, one, None, None, ws)
    torch.cuda.synchronize()
    assert torch.isfinite(one).all() and (one != 7.0).all()
    for at in range(0, n, 1 << 17):
        assert torch.equal(O[at:at + (1 << 17)], one[:, :1].expand(min(1 << 17, n - at), Hq, d)), at


def test_weights_of_many_rows():
    """W where the second launch needs more blocks than there are rows' tiles: 200 sequences, most of them short."""
    s = Serving(200, 4, 2, 32, 16, 40, "bf16")
    s.lengths[0] += dev_ints([600 if b % 50 == 7 else b % 23 for b in range(200)])
    W = s.weights(1.0)
    got = s.attend([1 + (b % 3) for b in range(200)], W=W, decay=0.5)
    s.check_attention(s.reference(), *got, W=W, W_before=np.full(W.shape, 1.0), decay=0.5)
