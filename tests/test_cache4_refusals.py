"""Arguments that the cache in 4 bits refuses, on the CPU: nothing is launched."""
import ctypes
import os
import re

import pytest
import torch

import cache4_ref as ref
import paper_2406_16747_amd as spk

ONE, ODD, NULL = ctypes.c_void_p(256), ctypes.c_void_p(264), ctypes.c_void_p(0)
BIG = 1 << 62


def ccfg(**kw):
    return spk.SparsekCache8Cfg(**{**dict(B=1, H=4, Hkv=2, d=64, cap=9, pages=18, format=spk.E2M1, dtype=spk.BF16, softmax_scale=1.0), **kw})


def struct(**kw):
    return spk.SparsekCache4(**{**{n: 256 for n, _ in spk.SparsekCache4._fields_}, **kw})


def calls(L, c, t):
    yield L.sparsek_cache4_append(c, t, ONE, NULL, 5, ONE, ONE, NULL)
    yield L.sparsek_cache4_read(c, t, ONE, 0, 5, ONE, ONE, NULL)
    yield L.sparsek_cache4_select(c, t, ONE, ONE, 4, ONE, NULL)
    yield L.sparsek_cache4_attn(c, t, ONE, ONE, ONE, 4, 0, ONE, ONE, ONE, BIG, NULL)
    yield L.sparsek_cache4_evict(c, t, ONE, 4, 1, 1, ctypes.c_void_p(1 << 20), ctypes.c_void_p(2 << 20), ctypes.c_void_p(3 << 20), NULL)


@pytest.mark.parametrize("kw,rc", [(x, -1) for x in (
    dict(B=0), dict(H=0), dict(Hkv=0), dict(H=5), dict(softmax_scale=0.0), dict(softmax_scale=float("inf")), dict(softmax_scale=float("nan")), dict(cap=0), dict(pages=0))] +
    [(x, -2) for x in (dict(d=32), dict(d=96), dict(dtype=spk.F32), dict(B=20000), dict(cap=8193), dict(pages=2 ** 24 + 1), dict(format=spk.I8), dict(format=spk.E4M3), dict(format=9))])
def test_configurations(kw, rc):
    L, c, t = spk.lib(), ccfg(**kw), struct()
    assert L.sparsek_cache4_attn_workspace_bytes(c, 0) == 0
    assert list(calls(L, c, t)) == [rc] * 5


def test_neither_cache_takes_the_other_s_format():
    L = spk.lib()
    t8 = spk.SparsekCache8(**{n: 256 for n, _ in spk.SparsekCache8._fields_})
    assert L.sparsek_cache8_append(ccfg(), t8, ONE, NULL, 5, ONE, ONE, NULL) == -2
    assert L.sparsek_cache8_attn_workspace_bytes(ccfg(), 0) == 0


def test_pointers():
    L, c, t = spk.lib(), ccfg(), struct()
    for name, _ in spk.SparsekCache4._fields_:
        assert list(calls(L, c, struct(**{name: 0}))) == [-1] * 5, name
    for name in ("k4", "v4", "ke", "ve", "km", "kt", "vt"):
        assert list(calls(L, c, struct(**{name: 264})))[:4] == [-1] * 4, name
    assert L.sparsek_cache4_append(c, None, ONE, NULL, 5, ONE, ONE, NULL) == -1
    assert L.sparsek_cache4_append(c, t, NULL, NULL, 5, ONE, ONE, NULL) == -1
    assert L.sparsek_cache4_append(c, t, ONE, NULL, 0, ONE, ONE, NULL) == -1
    assert L.sparsek_cache4_append(c, t, ONE, NULL, 5, ODD, ONE, NULL) == -1
    assert L.sparsek_cache4_append(c, t, ONE, NULL, 2 ** 30, ONE, ONE, NULL) == -2
    for args in ((None, ONE, 0, 5, ONE, ONE), (t, NULL, 0, 5, ONE, ONE), (t, ONE, -1, 5, ONE, ONE), (t, ONE, 0, 0, ONE, ONE), (t, ONE, 0, 5, NULL, ONE),
                 (t, ONE, 0, 5, ONE, NULL), (t, ONE, 0, 5, ODD, ONE), (t, ONE, 0, 5, ONE, ODD)):
        assert L.sparsek_cache4_read(c, *args, NULL) == -1
    assert L.sparsek_cache4_read(c, t, ONE, 2 ** 31 - 1, 2 ** 31 - 1, ONE, ONE, NULL) == -2
    assert L.sparsek_cache4_select(c, t, ONE, ONE, 0, ONE, NULL) == -1
    need = L.sparsek_cache4_attn_workspace_bytes(c, 4)
    assert need > 0 and L.sparsek_cache4_attn_workspace_bytes(c, -1) == 0
    assert L.sparsek_cache4_attn(c, t, ONE, ONE, ONE, 4, 0, ONE, ONE, ONE, need - 1, NULL) == -3
    assert L.sparsek_cache4_attn(c, t, ONE, ONE, NULL, 4, 0, ONE, ONE, ONE, BIG, NULL) == -1
    assert need == 256 and L.sparsek_cache4_attn_workspace_bytes(ccfg(cap=200), 0) > 256
    assert L.sparsek_cache4_attn(ccfg(cap=200), t, ONE, ONE, NULL, 0, 0, ONE, ONE, NULL, BIG, NULL) == -1
    far = [ctypes.c_void_p(x << 20) for x in (1, 2, 3)]
    for budget, sink, recent in ((-1, 0, 0), (4, 3, 2), (4, -1, 0), (4, 0, -1)):
        assert L.sparsek_cache4_evict(c, t, ONE, budget, sink, recent, *far, NULL) == -1
    assert L.sparsek_cache4_evict(c, t, ONE, 4, 1, 1, ONE, *far[1:], NULL) == -1


def test_the_binding_refuses_tensors_of_another_kind():
    cache = spk.Cache4.empty(1, 4, 2, 64, 4, device="cpu")
    k = torch.zeros(1, 2, 10, 64, dtype=torch.bfloat16)
    lens = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError):
        spk.Cache4.empty(1, 4, 2, 96, 4, device="cpu")
    for f in (lambda: spk.sparsek_cache4_append(cache, lens, k, k), lambda: spk.sparsek_cache4_append(cache, lens.long(), k, k),
              lambda: spk.sparsek_cache4_append(cache, lens, k.float(), k), lambda: spk.sparsek_cache4_read(cache, lens, 0, 5),
              lambda: spk.sparsek_cache4_read(cache, lens, 0, 5, out=(k, k)), lambda: cache.adopt(cache.table.long(), cache.mass),
              lambda: spk.sparsek_cache4_attn(cache, lens, k[:, :, 0])):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(AttributeError):
        cache.k4 = cache.v4


def test_the_reference_agrees_with_itself():
    """The two ways in which the reference rounds a block, and its page read back."""
    g = torch.Generator().manual_seed(1)
    for d in (64, 128):
        k, v = (torch.randn(64, d, generator=g) * torch.exp2(4 * torch.randn(64, d, generator=g))).bfloat16(), torch.randn(64, d, generator=g).bfloat16()
        k[3], v[:, 5] = 0.0, 2.0 ** -120
        k[7, 9], v[60, 11] = 3.3e38, -5e-35
        page = ref.page_bytes(k, v)
        cache = type("C", (), dict(d=d, k4=page[0][None], v4=page[1][None], ke=page[2][None], ve=page[3][None], ks=torch.ones(1), vs=torch.ones(1)))
        K, V = ref.dequantised(cache, 0)
        assert torch.equal(K, ref.rounded(k, -1)) and torch.equal(V, ref.rounded(v, -2))
        assert ((K - k.double()).abs() <= k.double().abs().view(64, -1, 32).amax(-1).repeat_interleave(32, 1) / 3 + 2.0 ** -100).all()


def test_every_entry_point_of_the_header_is_there():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sparsek.h")).read()
    names = set(re.findall(r"^(?:int|size_t) (sparsek_cache4_\w+)\(", header, re.M))
    assert len(names) == 6
    for name in names:
        assert getattr(spk.lib(), name), name


def test_reading_over_the_cache_or_itself():
    """(2 heads of 40 tokens of 64: 10240 bytes each.)  Outputs that lie over each other, or over what is read."""
    L, c = spk.lib(), ccfg()
    far = lambda x, more=0: ctypes.c_void_p((x << 32) + more)   # noqa: E731
    names = [n for n, _ in spk.SparsekCache4._fields_]
    t = spk.SparsekCache4(**{n: (x + 1) << 32 for x, n in enumerate(names)})
    k, v, lens = far(20), far(21), far(22)
    for more in (0, 16, 10224):
        assert L.sparsek_cache4_read(c, t, lens, 0, 40, k, far(20, more), NULL) == -1
        assert L.sparsek_cache4_read(c, t, lens, 0, 40, far(20, more), k, NULL) == -1
    for n in names:
        if n not in ("km", "kms", "mass"):   # (which reading does not look at)
            for more in (0, -10224):
                at = far(names.index(n) + 1, more)
                assert L.sparsek_cache4_read(c, t, lens, 0, 40, at, v, NULL) == -1, n
                assert L.sparsek_cache4_read(c, t, lens, 0, 40, k, at, NULL) == -1, n
    assert L.sparsek_cache4_read(c, t, lens, 0, 40, lens, v, NULL) == -1
