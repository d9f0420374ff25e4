"""Attention over the cache without weights in the workspace that it asks for then, of exactly that size."""
import pytest
import torch

import paper_2507_02957_amd as csat
from tests.gpu_harness import DEV
from tests.test_gpu_exact_attention import dev_ints
from tests.test_gpu_kv_cache import Serving

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,rows,capacity", [([5000, 0, 100], [1, 2, 1], 80), ([300, 7], [1, 5], 5), ([300, 40], [1, 1], 80)])
def test_without_weights(lens, rows, capacity, dtype):
    s = Serving(len(lens), 8, 2, 64, 64, capacity, dtype)
    s.lengths[0] += dev_ints(lens)
    Q, O, lse, off = s.attend(rows)
    again, l = torch.full_like(O, 7.0), torch.full_like(lse, 7.0)
    dims, cache = s.dims(Q.shape[0], 1, max(rows), 1), s.cache()
    n = csat.csat_cache_workspace_bytes_without_weights(dims, cache)
    assert n < csat.csat_cache_workspace_bytes(dims, cache)
    whole = torch.full((n + 4096,), 171, dtype=torch.uint8, device=DEV)
    csat.csat_cache_attention(dims, cache, Q, dev_ints(off), s.scale, 0.0, again, l, None, whole[:n] if n else None)
    torch.cuda.synchronize()
    assert torch.equal(again, O) and torch.equal(l, lse) and (whole[n:] == 171).all()
    s.check_attention(s.reference(), Q, again, l, off)
