"""The binding of the exact attention and its cache: tensors whose type or shape would make a call address memory outside them are refused
before the library sees them."""
import pytest
import torch

import paper_2507_02957_amd as csat

I32, F32 = torch.int32, torch.float32


def tensors(pages=3, heads=2, page=16, d=32, B=2, max_pages=2):
    return dict(K=torch.zeros(pages, heads, page, d, dtype=torch.uint8), V=torch.zeros(pages, heads, d, page, dtype=torch.uint8), Ks=torch.zeros(pages, heads),
                Vs=torch.zeros(pages, heads), table=torch.zeros(B, max_pages, dtype=I32), lengths=torch.zeros(B, dtype=I32))


@pytest.mark.parametrize("change", [
    dict(table=torch.zeros(2, 2, dtype=torch.int64)), dict(lengths=torch.zeros(2, dtype=torch.int64)), dict(lengths=torch.zeros(3, dtype=I32)),
    dict(Ks=torch.zeros(3, 2, dtype=torch.bfloat16)), dict(Vs=torch.zeros(2, 2)), dict(Vs=torch.zeros(3, 2, dtype=torch.float64)),
    dict(V=torch.zeros(3, 2, 16, 32, dtype=torch.uint8)), dict(V=torch.zeros(3, 2, 32, 32, dtype=torch.uint8)), dict(V=torch.zeros(2, 2, 32, 16, dtype=torch.uint8)),
    dict(K=torch.zeros(3, 2, 16, 32, dtype=torch.bfloat16)), dict(K=torch.zeros(3, 1, 16, 32, dtype=torch.uint8)), dict(K=torch.zeros(3, 2, 16, 64, dtype=torch.uint8)),
    dict(table=torch.zeros(2, 4, dtype=I32)[:, :2]), dict(K=torch.zeros(3, 2, 16, dtype=torch.uint8)), dict(table=torch.zeros(4, dtype=I32))])
def test_tensors_that_are_no_cache(change):
    csat.make_cache(**tensors())
    csat.make_cache(**{**tensors(), "K": tensors()["K"].view(torch.float8_e4m3fn)})
    with pytest.raises(ValueError):
        csat.make_cache(**{**tensors(), **change})


def calls(dims, cache, off=None, f=None, i=None, to=None):
    """The three calls with a cache; the tensors are of the host, so that none gets further than the binding."""
    x, off = torch.zeros(4, 2, 32, dtype=torch.bfloat16), torch.zeros(3, dtype=I32) if off is None else off
    f, i = torch.zeros(2, 2, 32) if f is None else f, torch.zeros(2, 2, 8, dtype=I32) if i is None else i
    return [lambda: csat.csat_cache_store(dims, cache, x, x, off), lambda: csat.csat_cache_attention(dims, cache, x, off, 1.0, 0.0, x, None, f, None),
            lambda: csat.csat_cache_evict(dims, cache, to or cache, f, f, 8, 0, i)]


def test_dims_that_are_not_the_caches():
    cache = csat.make_cache(**tensors())
    good = csat.make_packed_dims(2, 2, 2, 32, 4, 4, 2, 2, "bf16")
    for call in calls(good, cache):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
    for B, Hkv, d in ((3, 2, 32), (2, 1, 32), (2, 2, 16), (2, 2, 48)):
        for call in calls(csat.make_packed_dims(B, 2, Hkv, d, 4, 4, 2, 2, "bf16"), cache):
            with pytest.raises(ValueError, match="for a cache of"):
                call()
    with pytest.raises(ValueError, match="for a cache of"):
        calls(good, cache, to=csat.make_cache(**tensors(heads=1)))[2]()
    for call in calls(csat.make_packed_dims(1, 4, 2, 32, 4, 4, 2, 2, "bf16"), cache):      # the first sequence alone
        with pytest.raises(ValueError, match="on a GPU"):
            call()


def test_offsets_and_weights_of_other_types():
    cache, dims = csat.make_cache(**tensors()), csat.make_packed_dims(2, 2, 2, 32, 4, 4, 2, 2, "bf16")
    for call in calls(dims, cache, off=torch.zeros(3, dtype=torch.int64))[:2] + calls(dims, cache, f=torch.zeros(2, 2, 32, dtype=torch.bfloat16))[1:] + \
            calls(dims, cache, i=torch.zeros(2, 2, 8, dtype=torch.int64))[2:]:
        with pytest.raises(ValueError, match="is needed"):
            call()
    x, off = torch.zeros(4, 2, 32, dtype=torch.bfloat16), torch.zeros(3, dtype=I32)
    for q, k, lse in ((off.long(), off, None), (off, off.long(), None), (off, off, torch.zeros(2, 4, dtype=torch.bfloat16))):
        with pytest.raises(ValueError, match="is needed"):
            csat.csat_prompt_attention(dims, x, x, x, q, k, 1.0, x, lse, None)
