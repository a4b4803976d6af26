"""What block attention and the cache in 8 bits give out on the host: size queries, new caches.  On the CPU: nothing is launched."""
import pytest
import torch

import paper_2406_16747_amd as spk


@pytest.mark.parametrize("B,Hkv,cap,pages", [(2, 3, 5, None), (2, 3, 5, 30), (2, 3, 5, 100), (2, 3, 5, 29), (2, 3, 5, 12), (1, 1, 4, 3), (3, 2, 4, 5), (2, 1, 96, 96)])
def test_a_new_cache_has_no_page_in_two_places(B, Hkv, cap, pages):
    cache = spk.Cache8.empty(B, Hkv, Hkv, 64, cap, pages=pages, device="cpu")
    have = B * Hkv * cap if pages is None else pages
    assert cache.table.shape == (B, Hkv, cap) and cache.table.dtype is torch.int32 and cache.k8.shape[0] == have
    named = cache.table[cache.table >= 0].tolist()
    assert len(set(named)) == len(named) and all(x < have for x in named) and (cache.table >= -1).all()
    share = min(cap, have // (B * Hkv))
    assert (cache.table[..., :share] >= 0).all() and (cache.table[..., share:] == -1).all()
    if pages is None:
        assert cache.table.flatten().tolist() == list(range(have))


@pytest.mark.parametrize("kw", [dict(B=0), dict(Hkv=0, H=0), dict(cap=0), dict(pages=0), dict(pages=-3)])
def test_a_new_cache_of_nothing_is_refused(kw):
    with pytest.raises((ValueError, RuntimeError)):
        spk.Cache8.empty(**{**dict(B=1, H=4, Hkv=2, d=64, cap=4, device="cpu"), **kw})
