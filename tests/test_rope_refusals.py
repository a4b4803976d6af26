"""Arguments that the norms with rotary positions refuse, on the CPU: nothing is launched.  And the reference's gradients."""
import ctypes
import os
import re

import pytest
import torch

import paper_2406_16747_amd as spk
import rope_ref as ref

ODD, NULL = ctypes.c_void_p(264), ctypes.c_void_p(0)
BIG = 1 << 62


def far(x):
    return ctypes.c_void_p(x << 32)


def strides(*s):
    return spk.SparsekRopeStrides(*s)


def cfg(**kw):
    c = dict(B=2, H=4, Hkv=2, n=10, d=64, rot=64, axes=1, interleaved=0, norm=1, dtype=spk.BF16, eps=1e-6, q=strides(5120, 512, 64), k=strides(5120, 512, 64),
             dq=strides(5120, 512, 64), dk=strides(5120, 512, 64))
    return spk.SparsekRopeCfg(**{**c, **kw})


def calls(c, L=None):
    L = spk.lib()
    yield L.sparsek_rope_fwd(c, far(1), far(2), far(3), far(4), far(5), far(6), far(7), far(8), far(9), NULL)
    yield L.sparsek_rope_bwd(c, far(1), far(2), far(3), far(4), far(5), far(6), far(7), far(8), far(9), far(10), far(11), far(12), far(13), far(14), BIG, NULL)


@pytest.mark.parametrize("kw,rc", [(x, -1) for x in (
    dict(B=0), dict(H=0), dict(Hkv=-1), dict(n=0), dict(d=0), dict(rot=-8), dict(rot=72), dict(axes=0), dict(eps=0.0), dict(eps=1e-39), dict(eps=-1.0), dict(eps=float("nan")),
    dict(eps=float("inf")), dict(q=strides(-4, 512, 64)), dict(q=strides(5120, 510, 64)), dict(k=strides(2 ** 46, 512, 64)), dict(k=strides(5120, 2 ** 45, 64)))] +
    [(x, -2) for x in (dict(dtype=spk.I8), dict(d=60, rot=0), dict(d=264), dict(rot=12), dict(axes=5), dict(H=65535, Hkv=1), dict(B=65536, n=1025))])
def test_configurations(kw, rc):
    c = cfg(**kw)
    assert spk.lib().sparsek_rope_bwd_workspace_bytes(c) == 0
    assert list(calls(c)) == [rc] * 2


def test_pointers_and_workspaces():
    L, c = spk.lib(), cfg()
    need = L.sparsek_rope_bwd_workspace_bytes(c)
    assert need > 0 and L.sparsek_rope_fwd(None, *[far(1)] * 9, NULL) == -1
    for x in (0, 1, 2, 3, 7, 8):   # (axis and weights may be null)
        args = [far(y + 1) for y in range(9)]
        args[x] = NULL
        assert L.sparsek_rope_fwd(c, *args, NULL) == -1, x
        if x not in (2, 3):
            args[x] = ODD
            assert L.sparsek_rope_fwd(c, *args, NULL) == -1, x
    for x in (0, 1, 2, 3, 7, 8, 9, 10, 13):
        args = [far(y + 1) for y in range(14)]
        args[x] = NULL
        assert L.sparsek_rope_bwd(c, *args, BIG, NULL) == -1, x
        if x not in (2, 3):
            args[x] = ODD
            assert L.sparsek_rope_bwd(c, *args, BIG, NULL) == -1, x
    assert L.sparsek_rope_bwd(c, *[far(y + 1) for y in range(14)], need - 1, NULL) == -3
    # gradients of weights that have no part
    assert L.sparsek_rope_bwd(cfg(norm=0), *[far(y + 1) for y in range(14)], BIG, NULL) == -1
    assert L.sparsek_rope_bwd(cfg(Hkv=0), *[far(y + 1) for y in range(14)], BIG, NULL) == -1


def test_outputs_that_lie_over_inputs_or_themselves():
    L, c = spk.lib(), cfg()
    inputs, outputs = (0, 1), (7, 8)
    for x in inputs:
        for y in outputs:
            args = [far(z + 1) for z in range(9)]
            args[y] = ctypes.c_void_p(args[x].value + 16)
            assert L.sparsek_rope_fwd(c, *args, NULL) == -1
    args = [far(z + 1) for z in range(9)]
    args[8] = args[7]
    assert L.sparsek_rope_fwd(c, *args, NULL) == -1
    for x in (0, 1, 7, 8):
        for y in (9, 10):
            args = [far(z + 1) for z in range(14)]
            args[y] = ctypes.c_void_p(args[x].value + 16)
            assert L.sparsek_rope_bwd(c, *args, BIG, NULL) == -1
    args = [far(z + 1) for z in range(14)]
    args[10] = args[9]
    assert L.sparsek_rope_bwd(c, *args, BIG, NULL) == -1
    for s in (strides(5120, 512, 0), strides(0, 512, 64), strides(5120, 0, 64), strides(5120, 192, 64), strides(2048, 512, 64), strides(5120, 512, 60),
              strides(640, 64, 640)):
        assert L.sparsek_rope_bwd(cfg(dq=s), *[far(z + 1) for z in range(14)], BIG, NULL) == -1


def test_outputs_that_lie_over_what_goes_with_the_inputs():
    L, c = spk.lib(), cfg()
    for x in range(2, 7):
        for y in (7, 8):
            args = [far(z + 1) for z in range(9)]
            args[y] = ctypes.c_void_p(args[x].value + 16)
            assert L.sparsek_rope_fwd(c, *args, NULL) == -1, (x, y)
    for x in range(9):
        for y in range(9, 14):
            args = [far(z + 1) for z in range(14)]
            args[y] = args[x]
            assert L.sparsek_rope_bwd(c, *args, BIG, NULL) == -1, (x, y)
    for x in range(9, 14):
        for y in range(max(x + 1, 11), 14):
            args = [far(z + 1) for z in range(14)]
            args[y] = args[x]
            assert L.sparsek_rope_bwd(c, *args, BIG, NULL) == -1, (x, y)


def test_the_binding_refuses_tensors_of_another_kind():
    q, k = torch.zeros(1, 10, 4, 64, dtype=torch.bfloat16), torch.zeros(1, 10, 2, 64, dtype=torch.bfloat16)
    pos, freq, w = torch.zeros(1, 1, 10, dtype=torch.int32), torch.ones(32), torch.ones(64)
    for args, kw in (((q, k, pos, freq), {}),                                       # not on a GPU
                     ((q, k.float(), pos, freq), {}), ((q.half(), k.half(), pos, freq), {}), ((q[0], k, pos, freq), {}), ((q, k[:, :9], pos, freq), {}),
                     ((q.transpose(2, 3).contiguous().transpose(2, 3), k, pos, freq), {}), ((q, k, pos.long(), freq), {}), ((q, k, None, freq), {}),
                     ((q, k, pos[0], freq), {}), ((q, k, pos, freq.double()), {}), ((q, k, pos, freq), dict(axis=torch.zeros(31, dtype=torch.int32))),
                     ((q, k, pos, freq), dict(qw=w)), ((q, k, pos, freq), dict(norm=True, kw=w[:32])), ((q, k, pos, freq), dict(norm=True, qw=w.bfloat16()))):
        with pytest.raises((ValueError, TypeError)):
            spk.sparsek_rope_fwd(*args, **kw)
    go, gk = torch.zeros(1, 4, 10, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 10, 64, dtype=torch.bfloat16)
    for args, kw in (((q, k, pos, freq, go, gk), {}), ((q, k, pos, freq, go, None), {}), ((q, k, pos, freq, gk, go), {}), ((q, k, pos, freq, go.transpose(1, 2), gk), {}),
                     ((q, k, pos, freq, go, gk), dict(out=(q, None)))):
        with pytest.raises(ValueError):
            spk.sparsek_rope_bwd(*args, **kw)


@pytest.mark.parametrize("interleaved", [False, True])
def test_reference_gradients_against_differences(interleaved):
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)   # noqa: E731
    B, n, heads, d, rot = 2, 5, 3, 24, 16
    x, w, grad = rnd(B, n, heads, d), rnd(d), rnd(B, heads, n, d)
    pos, freq, axis = torch.randint(-50, 50, (2, B, n), generator=g, dtype=torch.int32), rnd(rot // 2).float(), torch.tensor([0, 1, 1, 0, 0, 1, 0, 1], dtype=torch.int32)
    dx, dw, _, _ = ref.bwd(x, pos, freq, axis, interleaved, True, w, 1e-6, grad)
    for what, got in ((x, dx), (w, dw)):
        step = rnd(*what.shape)
        L = []
        for sign in (1e-5, -1e-5):
            a, b = (x + sign * step, w) if what is x else (x, w + sign * step)
            L.append(float((ref.fwd(a, pos, freq, axis, interleaved, True, b, 1e-6)[0] * grad).sum()))
        want = (L[0] - L[1]) / 2e-5
        assert abs(float((got * step).sum()) - want) <= 1e-7 * (abs(want) + 1)


def test_every_entry_point_of_the_header_is_there():
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sparsek.h")).read()
    names = set(re.findall(r"^(?:int|size_t) (sparsek_rope_\w+)\(", header, re.M))
    assert len(names) == 3
    for name in names:
        assert getattr(spk.lib(), name), name
