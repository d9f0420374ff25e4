"""Store of sequences with more new rows than max_k: the first max_k of them at their own places, the other slots as they were."""
import pytest
import torch

import paper_2507_02957_amd as csat
from tests.gpu_harness import to_np
from tests.test_gpu_exact_attention import dev_ints, offsets
from tests.test_gpu_kv_cache import Serving

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,d", [(16, 32), (64, 128)])
@pytest.mark.parametrize("max_k", [1, 7, 16, 17, 70, 99])
def test_rows_beyond_the_bound(max_k, page, d, dtype):
    s = Serving(4, 2, 2, d, page, -(-160 // page), dtype)
    r = s.reference()
    s.store([20, 0, 33, 16], reference=r)
    lens, before = [100, 5, 0, 71], s.lengths[0].tolist()
    off = offsets(lens, 2)
    n = off[-1] + 1
    K, V = s.rows(n, 2, 30.0), s.rows(n, 2, 30.0)
    s.lengths[0] += dev_ints(lens)
    csat.csat_cache_store(s.dims(1, n, 1, max_k, K=K, V=V), s.cache(), K, V, dev_ints(off))
    torch.cuda.synchronize()
    t = s.tables[0].tolist()
    for b in range(4):
        for name, x in (("K", K), ("V", V)):
            r.store(name, t[b], before[b], to_np(x[off[b]:off[b] + min(lens[b], max_k)]).reshape(-1, 2, d))
    s.same_as(r)


def test_a_length_below_the_rows_is_not_stored_to():
    """... also where it is not below max_k."""
    s = Serving(2, 1, 1, 32, 16, 4, "bf16")
    r = s.reference()
    K = s.rows(20, 1)
    s.lengths[0] += dev_ints([9, 10])
    csat.csat_cache_store(s.dims(1, 20, 1, 4, K=K, V=K), s.cache(), K, K, dev_ints([0, 10, 20]))
    torch.cuda.synchronize()
    for name in "KV":
        r.store(name, s.tables[0][1].tolist(), 0, to_np(K[10:14]))
    s.same_as(r)
