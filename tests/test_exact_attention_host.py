"""Exact attention and the 8-bit cache: what is refused on the host, before anything touches the device."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paper_2507_02957_amd as csat
from tests import exact_reference as ref

P = ctypes.c_void_p(0x1000)            # aligned, non-NULL, never touched
ODD = ctypes.c_void_p(0x1004)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(csat.LIB_PATH):
        from paper_2507_02957_amd import build
        build.build()
    return csat.load_library()


def _dims(**kw):
    d = csat.make_packed_dims(2, 4, 2, 32, 10, 20, 8, 16, "bf16")
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def _cache(**kw):
    c = csat.csat_cache(8, 16, 3, 48, 0x1000, 0x1000, 0x1000, 0x1000, 0x1000, 0x1000)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_DIMS = [(dict(B=0), -2), (dict(Hq=3), -2), (dict(Hkv=0), -2), (dict(d=12), -2), (dict(d=264), -2), (dict(n_q=0), -2), (dict(n_k=-1), -2),
            (dict(max_q=0), -2), (dict(max_k=0), -2), (dict(dtype=7), -3), (dict(B=65536), -2), (dict(n_q=1 << 29), -2), (dict(n_k=(1 << 30) + 1), -2)]
BAD_CACHE = [(dict(pages=0), -2), (dict(page=48), -2), (dict(page=256), -2), (dict(page=8), -2), (dict(max_pages=0), -2), (dict(max_len=0), -2),
             (dict(max_len=49), -2), (dict(max_pages=1 << 28), -2)]
BAD_CACHE_POINTERS = [(dict([(k, None)]), -1) for k in ("K", "V", "Ks", "Vs", "table", "lengths")] + [(dict(K=0x1008), -4), (dict(table=0x1004), -4)]


def _prompt(lib, d, Q=P, K=P, V=P, qo=P, ko=P, scale=1.0, O=P, lse=None, ws=P, n=1 << 40, ctx=None):
    return lib.csat_prompt_attention(ctx or csat.context(), ctypes.byref(d), Q, K, V, qo, ko, scale, O, lse, ws, n, None)


def _store(lib, d, c, K=P, V=P, ko=P):
    return lib.csat_cache_store(csat.context(), ctypes.byref(d), ctypes.byref(c), K, V, ko, None)


def _attend(lib, d, c, Q=P, qo=P, scale=1.0, decay=0.0, O=P, lse=None, W=None, ws=P, n=1 << 40):
    return lib.csat_cache_attention(csat.context(), ctypes.byref(d), ctypes.byref(c), Q, qo, scale, decay, O, lse, W, ws, n, None)


P2 = ctypes.c_void_p(0x2000)


def _to(**kw):
    return _cache(**{**dict(table=0x2000, lengths=0x2000), **kw})


def _evict(lib, d, c, to, W=P, W_to=P2, budget=20, recent=4, kept=P):
    return lib.csat_cache_evict(csat.context(), ctypes.byref(d), ctypes.byref(c), ctypes.byref(to), W, W_to, budget, recent, kept, None)


@pytest.mark.parametrize("change,code", BAD_DIMS)
def test_dims_are_refused(lib, change, code):
    d, c = _dims(**change), _cache()
    n = ctypes.c_size_t()
    assert lib.csat_prompt_workspace_bytes(ctypes.byref(d), ctypes.byref(n)) == code
    assert lib.csat_cache_workspace_bytes(ctypes.byref(d), ctypes.byref(c), ctypes.byref(n)) == code
    assert _prompt(lib, d) == code and _store(lib, d, c) == code and _attend(lib, d, c) == code and _evict(lib, d, c, _to()) == code


@pytest.mark.parametrize("change,code", BAD_CACHE + BAD_CACHE_POINTERS)
def test_caches_are_refused(lib, change, code):
    d, c = _dims(), _cache(**change)
    n = ctypes.c_size_t()
    if (change, code) in BAD_CACHE:
        assert lib.csat_cache_workspace_bytes(ctypes.byref(d), ctypes.byref(c), ctypes.byref(n)) == code
    assert _store(lib, d, c) == code and _attend(lib, d, c) == code and _evict(lib, d, c, _to()) == code and _evict(lib, d, _cache(), _to(**change)) == code


def test_arguments_are_refused(lib):
    d, c = _dims(), _cache()
    n = ctypes.c_size_t()
    assert lib.csat_prompt_workspace_bytes(None, ctypes.byref(n)) == -1 and lib.csat_prompt_workspace_bytes(ctypes.byref(d), None) == -1
    assert lib.csat_cache_workspace_bytes(ctypes.byref(d), None, ctypes.byref(n)) == -1
    for name in ("Q", "K", "V", "qo", "ko", "O"):
        assert _prompt(lib, d, **{name: None}) == -1 and _prompt(lib, d, **{name: ODD}) == -4, name
    assert _prompt(lib, d, lse=ODD) == -4 and _prompt(lib, d, ws=ODD) == -4
    for name in ("K", "V", "ko"):
        assert _store(lib, d, c, **{name: None}) == -1 and _store(lib, d, c, **{name: ODD}) == -4, name
    for name in ("Q", "qo", "O"):
        assert _attend(lib, d, c, **{name: None}) == -1 and _attend(lib, d, c, **{name: ODD}) == -4, name
    assert _attend(lib, d, c, W=ODD) == -4 and _attend(lib, d, c, lse=ODD) == -4
    for name in ("W", "W_to", "kept"):
        assert _evict(lib, d, c, _to(), **{name: None}) == -1 and _evict(lib, d, c, _to(), **{name: ODD}) == -4, name
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _prompt(lib, d, scale=scale) == -6 and _attend(lib, d, c, scale=scale) == -6
    for decay in (-0.1, 1.1, float("nan")):
        assert _attend(lib, d, c, decay=decay) == -6
    assert _evict(lib, d, c, _to(), budget=0) == -6 and _evict(lib, d, c, _to(), recent=-1) == -6 and _evict(lib, d, c, _to(), recent=21) == -6
    assert _evict(lib, d, c, _to(max_len=19)) == -2 and _evict(lib, d, c, _to(page=32)) == -2
    # what other heads still read is not written over
    assert _evict(lib, d, c, _to(), W_to=P) == -6 and _evict(lib, d, c, _to(table=0x1000)) == -6 and _evict(lib, d, c, _to(lengths=0x1000)) == -6


@pytest.mark.parametrize("name,value", [(t + kind, v) for t in "qkvo" for kind, values in (("_token", (-8, 12, 1 << 24)), ("_head", (-8, 12))) for v in values])
def test_strides_are_refused(lib, name, value):
    d, c = _dims(**{name: value}), _cache()
    assert _prompt(lib, d) == -2
    if name[0] in "kv":
        assert _store(lib, d, c) == -2
    else:
        assert _attend(lib, d, c) == -2


def test_rows_of_the_output_that_overlap_are_refused(lib):
    for change in (dict(o_token=0), dict(o_head=0), dict(o_token=24), dict(o_head=24)):
        assert _prompt(lib, _dims(**change)) == -2 and _attend(lib, _dims(**change), _cache()) == -2


def _overlap(n, H, d, token, head):
    rows = sorted(i * token + h * head for i in range(n) for h in range(H))
    return any(b - a < d for a, b in zip(rows, rows[1:]))


def test_overlapping_rows_are_found_wherever_they_lie(lib):
    """All strides of a few rows and heads against their places; workspace of no bytes, so that none gets to the device."""
    seen = set()
    for token in range(32, 32 * 9, 8):
        for head in range(32, 32 * 12, 8):
            for n, H in ((3, 4), (10, 4), (2, 2), (7, 1), (1, 6)):
                d = _dims(n_q=n, Hq=H, Hkv=1, o_token=token, o_head=head, dtype=0)
                d.max_q, d.max_k, d.n_k = 1, 4096, 4096
                d.q_token, d.q_head = H * 32, 32
                bad = _overlap(n, H, 32, token, head)
                got = _prompt(lib, d, ws=None, n=0)
                assert got == (-2 if bad else -5), (token, head, n, H, got)
                seen.add(bad)
    assert seen == {False, True}



def test_tensors_of_the_host_are_refused(lib):
    x = torch.zeros(10, 4, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        csat.csat_prompt_attention(_dims(), x, x, x, x, x, 1.0, x, None, None)


def test_workspaces_are_refused(lib):
    d = _dims(n_q=1, max_q=1, n_k=100000, max_k=100000, B=1)       # one row, many keys: shares of them
    need = csat.csat_prompt_workspace_bytes(d)
    assert need > 0 and _prompt(lib, d, ws=None, n=0) == -5 and _prompt(lib, d, n=need - 1) == -5
    d, c = _dims(n_q=1, max_q=1, B=1), _cache(max_pages=10000, max_len=100000)
    need = csat.csat_cache_workspace_bytes(d, c)
    assert need > 0 and _attend(lib, d, c, ws=None, n=0) == -5 and _attend(lib, d, c, W=P, n=need - 1) == -5


def test_binding_takes_strides_and_keeps_tensors():
    x = torch.zeros(10, 8, 32, dtype=torch.bfloat16)
    d = csat.make_packed_dims(2, 4, 2, 32, 10, 10, 8, 8, torch.bfloat16, causal=False, Q=x[:, :4], K=x[:, 4:6], V=x[:, 6:])
    assert (d.q_token, d.q_head, d.k_token, d.v_token, d.o_token, d.o_head) == (256, 32, 256, 256, 128, 32) and d.causal == 0
    with pytest.raises(ValueError):
        csat.make_packed_dims(2, 4, 2, 32, 10, 10, 8, 8, "bf16", Q=x.transpose(1, 2))
    K = torch.zeros(3, 2, 16, 32, dtype=torch.uint8)
    V, s = K.transpose(2, 3).contiguous(), torch.zeros(3, 2)
    t, n = torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    c = csat.make_cache(K, V, s, s, t, n)
    assert (c.pages, c.page, c.max_pages, c.max_len) == (3, 16, 2, 32) and c.K == K.data_ptr() and c.lengths == n.data_ptr()
    assert csat.make_cache(K, V, s, s, t, n, 7).max_len == 7
    with pytest.raises(ValueError):
        csat.make_cache(K.transpose(2, 3), V, s, s, t, n)


def test_reference_rounds_like_torch():
    """The 64-bit e4m3 of the tests against torch's conversion, over all codes and the midpoints between them."""
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    fine = np.sort(codes[np.isfinite(codes)])
    x = np.concatenate([fine, (fine[1:] + fine[:-1]) / 2, fine * (1 + 2.0 ** -10), fine * (1 - 2.0 ** -10)])
    x = x[np.abs(x) <= 448]
    assert np.array_equal(ref.e4m3(x), torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy())
    assert ref.block_scale(np.array([448.0, np.inf])) == 1.0 and ref.block_scale(np.array([449.0])) == 2.0 and ref.block_scale(np.zeros(3)) == 2.0 ** -118
    assert ref.keep([1.0, 3.0, float("nan"), 3.0, 0.0, 0.5], 4, 1) == [1, 2, 3, 5]
