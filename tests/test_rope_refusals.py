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


def gradients(c, dk):
    """What a backward call says whose dk lies `dk` bytes behind dq; nothing is launched (the workspace is too small, which is looked at last)."""
    L = spk.lib()
    args = [far(z + 1) for z in range(14)]
    args[10] = ctypes.c_void_p(args[9].value + dk)
    return L.sparsek_rope_bwd(c, *args, L.sparsek_rope_bwd_workspace_bytes(c) - 1, NULL)


def beside(token, head_q, head_k, batch=None, **kw):
    return cfg(dq=strides(10 * token if batch is None else batch, token, head_q), dk=strides(10 * token if batch is None else batch, token, head_k), **kw)


@pytest.mark.parametrize("dtype,size", [(spk.BF16, 2), (spk.F32, 4)])
def test_gradients_of_queries_and_keys_in_one_tensor(dtype, size):
    """(2 sequences of 10 tokens, 4 + 2 heads of 64.)  Row beside row is allowed, rows over rows are not."""
    kw = dict(dtype=dtype)
    # slices of a fused gradient: 4 heads, 2 heads, 2 heads that belong to neither
    fused = beside(512, 64, 64, **kw)
    for at in (256, 320, 384):
        assert gradients(fused, at * size) == -3, at
    for at in (8, 56, 64, 192, 248, 392, 448, 504, 512, 512 + 64, 512 * 9 + 448, 512 * 9 + 504, 512 * 10 + 64, 512 * 19 + 192):
        assert gradients(fused, at * size) == -1, at
    for at in (512 + 256, 512 * 9 + 256, 512 * 10 + 384):     # (a row further on: the last rows lie behind the others)
        assert gradients(fused, at * size) == -3, at
    for at in (-128, -512 + 256, -512 * 10 + 384, -512 * 19 - 256, -512 * 19 + 256):
        assert gradients(fused, at * size) == -3, at
    for at in (-64, -120, -512 + 64, -512 * 10, -512 * 19 + 192):
        assert gradients(fused, at * size) == -1, at
    # a head's query, key and value beside each other
    three = beside(4 * 192, 192, 192, **kw)
    for at in (64, 72, 128, 192 + 64, 3 * 192 + 128):
        assert gradients(three, at * size) == -3, at
    for at in (8, 56, 136, 184, 192, 384):
        assert gradients(three, at * size) == -1, at
    # keys and values in turns behind the queries
    turns = beside(512, 64, 128, **kw)
    for at in (256, 320):
        assert gradients(turns, at * size) == -3, at
    for at in (0 + 8, 64, 128, 192, 248, 384, 392):
        assert gradients(turns, at * size) == -1, at
    # keys between the queries' groups
    groups = cfg(H=2, dq=strides(5120, 512, 256), dk=strides(5120, 512, 128), **kw)
    for at in (64, 448):
        assert gradients(groups, at * size) == -3, at
    for at in (128, 192 + 8, 384):
        assert gradients(groups, at * size) == -1, at
    # heads first, one block a sequence; and all of a tensor's tokens one sequence behind the other
    first = cfg(dq=strides(6 * 640, 64, 640), dk=strides(6 * 640, 64, 640), **kw)
    assert gradients(first, 4 * 640 * size) == -3 and gradients(first, (6 + 4) * 640 * size) == -3
    for at in (640, 3 * 640, 4 * 640 - 64, 4 * 640 - 8, 4 * 640 + 8, 5 * 640, 6 * 640):
        assert gradients(first, at * size) == -1, at
    # tokens first and heads first of one block a sequence
    mixed = cfg(dq=strides(6 * 640, 256, 64), dk=strides(6 * 640, 64, 640), **kw)
    assert gradients(mixed, 4 * 640 * size) == -3
    for at in (640, 4 * 640 - 8, 4 * 640 + 64):
        assert gradients(mixed, at * size) == -1, at
    # tensors of their own, and one sequence of one token
    assert gradients(cfg(dq=strides(2560, 256, 64), dk=strides(1280, 128, 64), **kw), 2 * 2560 * size) == -3
    one = cfg(B=1, n=1, dq=strides(0, 0, 64), dk=strides(0, 0, 64), **kw)
    assert gradients(one, 256 * size) == -3 and gradients(one, -128 * size) == -3
    for at in (8, 64, 192, 248, -64, -120):
        assert gradients(one, at * size) == -1, at


def test_gradients_in_one_tensor_against_every_place():
    """Small layouts, their places counted one by one: none is taken whose rows meet, and none refused whose strides are the same and whose rows do not."""
    g = torch.Generator().manual_seed(17)
    draw = lambda a, b: int(torch.randint(a, b + 1, (1,), generator=g))   # noqa: E731
    seen = {-1: 0, -3: 0}
    for case in range(3000):
        B, n, H, Hkv, d = draw(1, 3), draw(1, 5), draw(1, 4), draw(1, 4), 8 * draw(1, 3)

        def layout(heads):
            order = torch.randperm(3, generator=g).tolist()
            s, reach = [0, 0, 0], d
            for x in order:
                s[x] = reach + 4 * draw(0, 3) * draw(0, 12)
                reach = s[x] * ((B, n, heads)[x] - 1) + reach
            return s

        sq = layout(max(H, Hkv))
        sk = list(sq) if case % 3 else layout(Hkv)
        if case % 3 == 2 and sk[2] < min(sk[:2]):   # (heads nearer to each other, in the same tokens)
            sk[2] = draw(d, sk[2]) // 4 * 4
        c = cfg(B=B, n=n, H=H, Hkv=Hkv, d=d, rot=0, dtype=spk.F32, dq=strides(*sq), dk=strides(*sk))
        rows = lambda s, heads: [b * s[0] + t * s[1] + h * s[2] for b in range(B) for t in range(n) for h in range(heads)]   # noqa: E731
        q, k = sorted(rows(sq, H)), sorted(rows(sk, Hkv))
        if any(y - x < d for x, y in zip(k, k[1:])):
            continue
        at = 4 * draw(-(k[-1] + d) // 4, (q[-1] + d) // 4)
        places = torch.zeros(max(q[-1], k[-1]) + abs(at) + d + 1, dtype=torch.int8)
        for x in q:
            places[x + max(-at, 0):x + max(-at, 0) + d] = 1
        meet = any(bool(places[x + max(at, 0):x + max(at, 0) + d].any()) for x in k)
        rc = gradients(c, 4 * at)
        seen[rc] += 1
        assert rc == (-1 if meet else -3), (B, n, H, Hkv, d, sq, sk, at)
    assert min(seen.values()) > 300
