"""Sizes at the limits that csat.h states, and queries that refuse what a call refuses."""
import ctypes

import pytest

from tests.test_exact_attention_host import P, _attend, _cache, _dims, _evict, _prompt, _store, _to, lib  # noqa: F401


def _query(lib, name, d, c=None):  # noqa: F811
    n = ctypes.c_size_t()
    args = [ctypes.byref(d)] + ([ctypes.byref(c)] if c is not None else []) + [ctypes.byref(n)]
    return getattr(lib, name)(*args), n.value


@pytest.mark.parametrize("rows,heads,d", [(131072, 32, 128), (1 << 24, 64, 16), (1 << 20, 1024, 256), (1 << 30, 1, 16)])
def test_many_rows_over_the_cache_are_taken(lib, rows, heads, d):  # noqa: F811
    """... with a workspace of no bytes, so that none gets to the device."""
    dims = _dims(B=1, Hq=heads, Hkv=1, d=d, n_q=rows, max_q=rows, q_token=heads * d if heads * d < 1 << 24 else d, q_head=d, o_token=heads * d if heads * d < 1 << 24 else d, o_head=d)
    c = _cache(max_pages=100, max_len=1600)
    status, need = _query(lib, "csat_cache_workspace_bytes_without_weights", dims, c)
    assert status == 0 and need > 0 and _attend(lib, dims, c, ws=None, n=0) == -5 and _attend(lib, dims, c, n=need - 1) == -5


def test_scores_beyond_any_memory_are_refused(lib):  # noqa: F811
    """Their size is no 64-bit number, or wraps to a small one: the query and the call say so."""
    for B, rows, heads, pages in ((65535, 1 << 24, 64, 4096), (1024, 1 << 30, 1, 1 << 20), (4096, 1 << 24, 64, 1 << 16)):
        d = _dims(B=B, Hq=heads, Hkv=1, n_q=rows, max_q=rows, q_token=heads * 32, q_head=32, o_token=heads * 32, o_head=32)
        c = _cache(max_pages=pages, max_len=16 * pages)
        assert _query(lib, "csat_cache_workspace_bytes", d, c)[0] == -2
        assert _attend(lib, d, c, W=P, n=1 << 60) == -2
        assert _query(lib, "csat_cache_workspace_bytes_without_weights", d, c)[0] == 0


def test_stated_limits(lib):  # noqa: F811
    for d, c, code in ((_dims(B=65535, Hq=64, Hkv=64), _cache(), 0), (_dims(B=65535, Hq=65, Hkv=65), _cache(), -2),
                       (_dims(), _cache(max_pages=(1 << 20) - 1, max_len=16 * ((1 << 20) - 1)), 0), (_dims(), _cache(max_pages=1 << 20, max_len=1 << 24), -2),
                       (_dims(Hkv=1), _cache(page=128, max_pages=(1 << 21) - 1, max_len=128 * ((1 << 21) - 1)), 0)):
        assert _query(lib, "csat_cache_workspace_bytes_without_weights", d, c)[0] == code, (d.B, c.max_pages)
        if code:
            assert _attend(lib, d, c) == code and _store(lib, d, c) == code and _evict(lib, d, c, _to()) == code
        if d.B == 65535:
            assert _query(lib, "csat_prompt_workspace_bytes", d)[0] == code and (not code or _prompt(lib, d) == code)
    d = _dims(B=1024, Hq=4, Hkv=4)
    assert _evict(lib, d, _cache(), _to(), budget=(1 << 18) + 1) == -2              # (1024 x 4 x 2^18 = 2^30 is the most)


def test_scales_that_are_no_float_in_units_of_log2_are_refused(lib):  # noqa: F811
    """Scores are formed as scale log2(e) q.k: above 2^127 that factor is infinite, and 0 times it no number."""
    d, c = _dims(), _cache()
    for scale in (1.8e38, 2.4e38, 3.4e38):
        assert _prompt(lib, d, scale=scale) == -6 and _attend(lib, d, c, scale=scale) == -6
    few = _dims(n_q=1, max_q=1, n_k=100000, max_k=100000, B=1)                       # (2^127 itself gets to the workspace's check)
    assert _prompt(lib, few, scale=2.0 ** 127, ws=None, n=0) == -5 and _attend(lib, few, _cache(max_pages=10000, max_len=100000), scale=2.0 ** 127, ws=None, n=0) == -5
