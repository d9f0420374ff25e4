"""How much workspace attention over the cache asks for, with and without the tokens' weights."""
import ctypes

import pytest

import paper_2507_02957_amd as csat
from tests.test_exact_attention_host import BAD_CACHE, BAD_DIMS, P, _attend, _cache, _dims, lib  # noqa: F401


@pytest.mark.parametrize("change,code", BAD_DIMS)
def test_dims_are_refused(lib, change, code):  # noqa: F811
    d, c, n = _dims(**change), _cache(), ctypes.c_size_t()
    assert lib.csat_cache_workspace_bytes_without_weights(ctypes.byref(d), ctypes.byref(c), ctypes.byref(n)) == code


@pytest.mark.parametrize("change,code", BAD_CACHE)
def test_caches_are_refused(lib, change, code):  # noqa: F811
    d, c, n = _dims(), _cache(**change), ctypes.c_size_t()
    assert lib.csat_cache_workspace_bytes_without_weights(ctypes.byref(d), ctypes.byref(c), ctypes.byref(n)) == code


def test_nothing_to_write_to_is_refused(lib):  # noqa: F811
    d, c, n = _dims(), _cache(), ctypes.c_size_t()
    query = lib.csat_cache_workspace_bytes_without_weights
    assert query(None, ctypes.byref(c), ctypes.byref(n)) == -1 and query(ctypes.byref(d), None, ctypes.byref(n)) == -1 and query(ctypes.byref(d), ctypes.byref(c), None) == -1


@pytest.mark.parametrize("B,rows,Hq,Hkv,d,max_len,dtype", [(64, 1, 32, 8, 128, 131072, "bf16"), (1, 512, 32, 8, 128, 131072, "bf16"), (1, 1, 8, 2, 64, 300, "bf16"),
                                                         (3, 2, 4, 1, 256, 5000, "f32")])
def test_scores_are_asked_for_only_with_weights(lib, B, rows, Hq, Hkv, d, max_len, dtype):  # noqa: F811
    dims = csat.make_packed_dims(B, Hq, Hkv, d, B * rows, 1, rows, 1, dtype)
    c = _cache(pages=100, page=64, max_pages=-(-max_len // 64), max_len=max_len)
    scores = B * rows * Hq * (-(-max_len // 64) * 64) * 4
    plain, weighted = csat.csat_cache_workspace_bytes_without_weights(dims, c), csat.csat_cache_workspace_bytes(dims, c)
    assert weighted - plain >= scores
    parts = 0 if max_len <= 512 else plain                        # one share: nothing to join
    assert plain == parts and plain <= 512 * B * rows * Hq * (d + 2) * 4
    if plain:
        assert _attend(lib, dims, c, ws=None, n=0) == -5 and _attend(lib, dims, c, n=plain - 1) == -5
    assert _attend(lib, dims, c, W=P, n=plain) == -5 and _attend(lib, dims, c, W=P, n=weighted - 1) == -5
