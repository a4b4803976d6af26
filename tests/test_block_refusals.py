"""Arguments that the block attention and the cache in 8 bits refuse, on the CPU: nothing is launched."""
import ctypes
import json
import os
import re

import pytest
import torch

import block_ref as ref
import paper_2406_16747_amd as spk

ONE, ODD, NULL = ctypes.c_void_p(256), ctypes.c_void_p(264), ctypes.c_void_p(0)
BIG = 1 << 62


def bcfg(**kw):
    return spk.SparsekBlockCfg(**{**dict(B=1, H=4, Hkv=2, n=300, d=64, top=3, dtype=spk.BF16, softmax_scale=1.0), **kw})


def ccfg(**kw):
    return spk.SparsekCache8Cfg(**{**dict(B=1, H=4, Hkv=2, d=64, cap=9, pages=18, format=spk.I8, dtype=spk.BF16, softmax_scale=1.0), **kw})


INVALID = [dict(B=0), dict(H=0), dict(Hkv=0), dict(H=5), dict(softmax_scale=0.0), dict(softmax_scale=float("inf")), dict(softmax_scale=float("nan"))]
UNSUPPORTED = [dict(d=32), dict(d=96), dict(d=0), dict(dtype=spk.F32), dict(B=20000), dict(H=2 ** 30, Hkv=2 ** 30)]


@pytest.mark.parametrize("kw,rc", [(x, -1) for x in INVALID + [dict(n=0), dict(n=-1), dict(top=-1)]] +
                         [(x, -2) for x in UNSUPPORTED + [dict(n=2 ** 20 + 1), dict(top=65), dict(H=4096, Hkv=1, n=2 ** 20)]])
def test_block_configurations(kw, rc):
    L, c = spk.lib(), bcfg(**kw)
    for name in ("select", "attn_fwd", "attn_bwd"):
        assert getattr(L, "sparsek_block_%s_workspace_bytes" % name)(c) == 0
    assert L.sparsek_block_select(c, ONE, ONE, ONE, ONE, BIG, NULL) == rc
    assert L.sparsek_block_attn_fwd(c, *[ONE] * 7, ONE, BIG, NULL) == rc
    assert L.sparsek_block_attn_bwd(c, *[ONE] * 10, ONE, BIG, NULL) == rc


def test_block_pointers_and_workspaces():
    L, c = spk.lib(), bcfg()
    calls = (("sparsek_block_select", 4, (0, 1, 3)), ("sparsek_block_attn_fwd", 8, (0, 1, 2, 4, 7)), ("sparsek_block_attn_bwd", 11, (0, 1, 2, 4, 6, 7, 8, 9, 10)))
    for name, count, wide in calls:
        f = getattr(L, name)
        need = getattr(L, name + "_workspace_bytes")(c)
        assert need > 0
        for x in range(count):
            if name == "sparsek_block_attn_fwd" and x == 6:
                continue   # mass may be null
            args = [ONE] * count
            args[x] = NULL
            assert f(c, *args, BIG, NULL) == -1, (name, x)
            if x in wide:
                args[x] = ODD
                assert f(c, *args, BIG, NULL) == -1, (name, x)
        assert f(c, *[ONE] * count, need - 1, NULL) == -3
    assert L.sparsek_block_select(None, ONE, ONE, ONE, ONE, BIG, NULL) == -1
    # sizes of long documents do not wrap: the backward's partial results of a million tokens, the forward's of one stretch
    big = bcfg(H=32, Hkv=8, d=128, n=2 ** 20, top=16)
    assert L.sparsek_block_attn_bwd_workspace_bytes(big) > 2 ** 37
    assert 2 ** 33 < L.sparsek_block_attn_fwd_workspace_bytes(big) < 2 ** 35


def cache_struct(**kw):
    return spk.SparsekCache8(**{**{n: 256 for n in ("k8", "v8", "ks", "vs", "km", "kms", "kt", "vt", "table", "mass")}, **kw})


def cache_calls(L, c, t):
    yield L.sparsek_cache8_append(c, t, ONE, NULL, 5, ONE, ONE, NULL)
    yield L.sparsek_cache8_select(c, t, ONE, ONE, 4, ONE, NULL)
    yield L.sparsek_cache8_attn(c, t, ONE, ONE, ONE, 4, 0, ONE, ONE, ONE, BIG, NULL)
    yield L.sparsek_cache8_evict(c, t, ONE, 4, 1, 1, ctypes.c_void_p(1 << 20), ctypes.c_void_p(2 << 20), ctypes.c_void_p(3 << 20), NULL)


@pytest.mark.parametrize("kw,rc", [(x, -1) for x in INVALID + [dict(cap=0), dict(pages=0)]] +
                         [(x, -2) for x in UNSUPPORTED + [dict(cap=8193), dict(pages=2 ** 24 + 1), dict(format=spk.F32), dict(format=9)]])
def test_cache_configurations(kw, rc):
    L, c, t = spk.lib(), ccfg(**kw), cache_struct()
    assert L.sparsek_cache8_attn_workspace_bytes(c, 0) == 0
    assert list(cache_calls(L, c, t)) == [rc] * 4


def test_cache_pointers():
    L, c, t = spk.lib(), ccfg(), cache_struct()
    for name, _ in spk.SparsekCache8._fields_:
        assert list(cache_calls(L, c, cache_struct(**{name: 0}))) == [-1] * 4, name
    for name in ("k8", "v8", "km", "kt", "vt"):
        assert list(cache_calls(L, c, cache_struct(**{name: 264})))[:3] == [-1] * 3, name
    assert L.sparsek_cache8_append(c, None, ONE, NULL, 5, ONE, ONE, NULL) == -1
    assert L.sparsek_cache8_append(c, t, NULL, NULL, 5, ONE, ONE, NULL) == -1
    assert L.sparsek_cache8_append(c, t, ONE, NULL, 0, ONE, ONE, NULL) == -1
    assert L.sparsek_cache8_append(c, t, ONE, NULL, 5, ODD, ONE, NULL) == -1
    assert L.sparsek_cache8_append(c, t, ONE, NULL, 2 ** 30, ONE, ONE, NULL) == -2
    assert L.sparsek_cache8_select(c, t, ONE, ONE, 0, ONE, NULL) == -1
    assert L.sparsek_cache8_select(c, t, ONE, ONE, 2 ** 30, ONE, NULL) == -2
    need = L.sparsek_cache8_attn_workspace_bytes(c, 4)
    assert need > 0 and L.sparsek_cache8_attn_workspace_bytes(c, -1) == 0
    assert L.sparsek_cache8_attn(c, t, ONE, ONE, ONE, 4, 0, ONE, ONE, ONE, need - 1, NULL) == -3
    assert L.sparsek_cache8_attn(c, t, ONE, ONE, NULL, 4, 0, ONE, ONE, ONE, BIG, NULL) == -1
    assert L.sparsek_cache8_attn(c, t, ONE, ONE, ONE, 0, 0, ONE, ONE, ONE, BIG, NULL) == -1
    far = [ctypes.c_void_p(x << 20) for x in (1, 2, 3)]
    for budget, sink, recent in ((-1, 0, 0), (4, 3, 2), (4, -1, 0), (4, 0, -1), (4, 2 ** 31 - 1, 2 ** 31 - 1)):
        assert L.sparsek_cache8_evict(c, t, ONE, budget, sink, recent, *far, NULL) == -1
    for x in range(3):   # an output where an input, or another output, is
        for y in (ctypes.c_void_p(256), far[(x + 1) % 3]):
            out = list(far)
            out[x] = y
            assert L.sparsek_cache8_evict(c, t, ONE, 4, 1, 1, *out, NULL) == -1


def test_the_binding_refuses_tensors_of_another_kind():
    q, k = torch.zeros(1, 4, 100, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 100, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        spk.sparsek_block_select(q, k, 2)                      # not on a GPU
    with pytest.raises(ValueError):
        spk.sparsek_block_select(q.float(), k, 2)
    with pytest.raises(ValueError):
        spk.sparsek_block_select(q, k[:, :, :99], 2)
    with pytest.raises(ValueError):
        spk.sparsek_block_select(q.transpose(1, 2).contiguous().transpose(1, 2), k, 2)
    with pytest.raises(ValueError):
        spk.sparsek_block_attn_fwd(q, k, k, torch.zeros(1, 2, 100, 3), 1.0)
    with pytest.raises(ValueError):
        spk.Cache8.empty(1, 4, 2, 96, 4, device="cpu")
    cache = spk.Cache8.empty(1, 4, 2, 64, 4, device="cpu")
    with pytest.raises(ValueError):
        cache.adopt(cache.table.long(), cache.mass)
    with pytest.raises(ValueError):
        spk.sparsek_cache8_append(cache, torch.zeros(1, dtype=torch.int64), k, k)


def test_reference_gradients_against_differences():
    """The formulas that the kernels are held to, against central differences of the forward's definition."""
    g = torch.Generator().manual_seed(3)
    B, H, Hkv, n, d, scale = 1, 4, 2, 150, 8, 0.4
    q, k, v, dO = (torch.randn(B, h, n, d, generator=g, dtype=torch.float64) for h in (H, Hkv, Hkv, H))
    idx = torch.randint(-1, 3, (B, Hkv, n, 2), generator=g, dtype=torch.int32)
    o, lse = ref.attn(q, k, v, idx, scale)[:2]
    grads, _ = ref.attn_bwd(q, k, v, idx, o, lse, dO, scale)
    for which in range(3):
        x = (q, k, v)[which]
        step = torch.randn(x.shape, generator=g, dtype=torch.float64)
        L = []
        for sign in (1, -1):
            args = [q, k, v]
            args[which] = x + sign * 1e-5 * step
            L.append(float((ref.attn(*args, idx, scale)[0] * dO).sum()))
        want = (L[0] - L[1]) / 2e-5
        assert abs(float((grads[which] * step).sum()) - want) <= 1e-7 * (abs(want) + 1)


def test_every_entry_point_of_the_header_is_there():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sparsek.h")).read()
    names = set(re.findall(r"^(?:int|size_t) (sparsek_(?:block|cache8)_\w+)\(", header, re.M))
    assert len(names) == 11
    for name in names:
        assert getattr(spk.lib(), name), name


def test_hand_written_m0_is_checked():
    """The kernels whose direct-to-LDS loads set M0 by hand (like those that test_abi.py lists) went through the build's check."""
    from paper_2406_16747_amd import build

    if not os.path.exists(build.SIDECAR) or os.path.getmtime(build.SIDECAR) < os.path.getmtime(spk.lib_path()) - 60:
        build.build()
    rec = json.load(open(build.SIDECAR))
    assert rec["m0_check"] == "ok" and set(rec["untracked_direct_to_lds_loads_of_blocks"]) == {"block_attn_bwd.hip", "cache8.hip"}
