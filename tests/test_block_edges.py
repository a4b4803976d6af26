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


@pytest.mark.parametrize("n", [1, 63, 64, 65])
@pytest.mark.parametrize("top", [0, 1, 64])
def test_every_configuration_that_is_served_has_a_workspace(n, top):
    """0 stands for a configuration that is refused."""
    c = spk.SparsekBlockCfg(B=1, H=2, Hkv=1, n=n, d=64, top=top, dtype=spk.BF16, softmax_scale=1.0)
    for name in ("select", "attn_fwd", "attn_bwd"):
        assert getattr(spk.lib(), "sparsek_block_%s_workspace_bytes" % name)(c) > 0, name
