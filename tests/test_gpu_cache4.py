"""The key/value cache in blocks held in 4 bits: what goes in, reading it back, the single-token attention over it, selection and eviction,
against their definitions in 64 bits."""
import pytest
import torch

import block_ref
import cache4_ref as ref
import paper_2406_16747_amd as spk
import rope_ref
from gpu_util import require_gpu, say

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator().manual_seed(seed)


def rand(g, *s):
    return torch.randn(*s, generator=g).bfloat16().cuda()


def ints(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def shuffled(cache, seed):
    n = cache.table.numel()
    cache.table.copy_(torch.randperm(n, generator=gen(seed)).to(torch.int32).view(cache.table.shape))
    return cache


def filled(seed, lens, H, Hkv, d, cap=None, scale=None):
    B, c = len(lens), max(max(lens), 1)
    cache = shuffled(spk.Cache4.empty(B, H, Hkv, d, cap or c // 64 + 1, scale=scale), seed)
    g = gen(seed)
    k, v = rand(g, B, Hkv, c, d), rand(g, B, Hkv, c, d)
    L = ints(lens)
    spk.sparsek_cache4_append(cache, torch.zeros_like(L), k, v, counts=L)
    return cache, L, k, v


def given(k, v, H, cap, scale=None):
    """A cache with all of k, v [B,Hkv,n,d] in it, and its lengths."""
    B, Hkv, n, d = k.shape
    cache = spk.Cache4.empty(B, H, Hkv, d, cap, scale=scale)
    spk.sparsek_cache4_append(cache, torch.zeros(B, dtype=torch.int32).cuda(), k, v)
    return cache, ints([n] * B)


def as_held(x, n, dim):
    """[Hkv, c, d] -> the n tokens as the cache holds them, in 64 bits."""
    whole = n // 64 * 64
    y = ref.f64(x[:, :n]).clone()
    if whole:
        y[:, :whole] = ref.rounded(x[:, :whole].unflatten(1, (-1, 64)), dim).flatten(1, 2)
    return y


def same(a, b):
    """Equal, or both NaN."""
    return bool(((a == b) | (a.isnan() & b.isnan())).all())


@pytest.mark.parametrize("d,pieces", [(64, [1]), (128, [63, 1]), (64, [64, 64]), (128, [40, 100, 1, 1, 300]), (64, [10, 117, 1, 64, 200]), (128, [127, 1])])
def test_append_in_pieces(d, pieces):
    """The bytes of every page are where the header says, whatever the pieces; reading gives the values back."""
    require_gpu()
    say("cache4 append", d, pieces)
    B, Hkv, n = 2, 2, sum(pieces)
    cache = shuffled(spk.Cache4.empty(B, Hkv, Hkv, d, n // 64 + 1), 3)
    g = gen(1)
    k, v = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d)
    lens = torch.zeros(B, dtype=torch.int32).cuda()
    for c in pieces:
        a = int(lens[0])
        spk.sparsek_cache4_append(cache, lens, k[:, :, a:a + c].contiguous(), v[:, :, a:a + c].contiguous())
        lens += c
    rk, rv = spk.sparsek_cache4_read(cache, lens, 0, n)
    torch.cuda.synchronize()
    for b in range(B):
        assert torch.equal(ref.f64(rk[b]), as_held(k[b], n, -1)) and torch.equal(ref.f64(rv[b]), as_held(v[b], n, -2))
        for h in range(Hkv):
            for j in range(n // 64):
                page = int(cache.table[b, h, j])
                kb, vb = k[b, h, 64 * j:64 * j + 64], v[b, h, 64 * j:64 * j + 64]
                if j < 2:
                    for got, want in zip((cache.k4, cache.v4, cache.ke, cache.ve), ref.page_bytes(kb, vb)):
                        assert torch.equal(got[page].cpu(), want), (b, h, j)
                assert float(cache.ks[page]) == ref.page_scale(cache.ke[page].cpu()) and float(cache.vs[page]) == ref.page_scale(cache.ve[page].cpu())
                y, s = ref.mean_codes(kb)
                assert torch.equal(cache.km[page].cpu().float(), y) and float(cache.kms[page]) == float(s), (b, h, j)
            rest = n % 64
            assert torch.equal(cache.kt[b, h, :rest], k[b, h, n - rest:n]) and torch.equal(cache.vt[b, h, :, :rest], v[b, h, n - rest:n].T)


def test_append_of_padded_prompts():
    """Counts of nothing, of some and of all; what lies behind a sequence's last token stays as it was."""
    require_gpu()
    say("cache4 append, padded")
    lens = [0, 1, 64, 200, 131]
    cache, L, k, v = filled(5, lens, 4, 2, 64)
    rk, rv = spk.sparsek_cache4_read(cache, L, 0, 230)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        assert torch.equal(ref.f64(rk[b, :, :n]), as_held(k[b], n, -1)) and torch.equal(ref.f64(rv[b, :, :n]), as_held(v[b], n, -2))
        assert (rk[b, :, n:] == 0).all() and (rv[b, :, n:] == 0).all()
        assert (cache.kt[b, :, n % 64:] == 0).all() and (cache.vt[b, :, :, n % 64:] == 0).all()
        for h in range(2):
            rest = cache.table[b, h, n // 64:].long()
            assert (cache.ks[rest] == 0).all() and (cache.k4[rest] == 0).all() and (cache.km[rest] == 0).all() and (cache.ve[rest] == 0).all()


def test_counts_lengths_and_pages_out_of_range():
    """Everything else stays as it was, and what is read there is zeros."""
    require_gpu()
    say("cache4, out of range")
    g = gen(9)
    cache = spk.Cache4.empty(4, 2, 2, 64, 2, pages=8)
    cache.table[0, 0, 0], cache.table[0, 1, 0] = -1, 8
    cache.table[0, :, 1] = 2 ** 31 - 1
    cache.table[1:] = torch.arange(12, dtype=torch.int32).view(3, 2, 2).cuda() % 4 + 4
    k, v = rand(g, 4, 2, 300, 64), rand(g, 4, 2, 300, 64)
    lens, counts = ints([0, 191, 2 ** 31 - 1, -5]), ints([300, 300, 2 ** 31 - 1, -1])
    spk.sparsek_cache4_append(cache, lens, k, v, counts=counts)
    torch.cuda.synchronize()
    assert (cache.k4 == 0).all() and (cache.ks == 0).all() and (cache.ke == 0).all()   # 0: bad pages; 1 and 2: full; 3: no tokens
    assert torch.equal(cache.kt[0, :, :63], k[0, :, 128:191])                           # 191 of 300 fit
    assert (cache.kt[1:] == 0).all() and (cache.kt[0, :, 63] == 0).all()
    rk, rv = spk.sparsek_cache4_read(cache, ints([300, 2 ** 31 - 1, -5, 0]), 100, 150)
    torch.cuda.synchronize()
    assert torch.equal(rk[0, :, 28:91], k[0, :, 128:191]) and torch.equal(rv[0, :, 28:91], v[0, :, 128:191])
    assert (rk[0, :, :28] == 0).all() and (rk[0, :, 91:] == 0).all() and (rk[1:] == 0).all() and (rv[1:] == 0).all()


@pytest.mark.parametrize("kind", ["zeros", "tiny", "one value", "largest", "wide", "ties"])
@pytest.mark.parametrize("d", [64, 128])
def test_blocks_of_all_kinds(kind, d):
    """What is read is the definition's, and so is the attention, over groups of every size beside each other."""
    require_gpu()
    say("cache4 blocks,", kind, d)
    g = gen(4)
    k, v = rand(g, 1, 2, 130, d), rand(g, 1, 2, 130, d)
    for x in (k, v):
        if kind == "zeros":
            x[:, :, :64] = 0
        elif kind == "tiny":
            x[:, 0, :64] *= 2.0 ** -110
            x[:, 1, :32] *= 2.0 ** -104
        elif kind == "one value":
            x[:, :, :64] = -3.0
        elif kind == "largest":
            x[:, :, 5, 7] = 3.3e38
            x[:, :, 6, 40] = -2.6e38
        elif kind == "wide":   # tokens and channels from 2^-60 to 2^30
            x[:, 0, :64] *= torch.exp2(torch.arange(64).float() * 90 / 64 - 60).view(64, 1).cuda().bfloat16()
            x[:, 1, :64] *= torch.exp2(torch.arange(d).float().flip(0) * 90 / d - 60).cuda().bfloat16()
        else:                  # halves between codes, of both signs, and a group whose largest is one and a half times a power of two
            x[:, :, :64] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0] * (d // 16)).cuda().bfloat16()
            x[:, :, 32:64] *= 2.0
    cache, L = given(k, v, 4, 3)
    rk, rv = spk.sparsek_cache4_read(cache, L, 0, 130)
    torch.cuda.synchronize()
    for h in range(2):
        assert torch.equal(ref.f64(rk[0]), as_held(k[0], 130, -1)) and torch.equal(ref.f64(rv[0]), as_held(v[0], 130, -2))
        for j in range(2):
            page = int(cache.table[0, h, j])
            assert float(cache.ks[page]) == ref.page_scale(cache.ke[page].cpu()) and float(cache.vs[page]) == ref.page_scale(cache.ve[page].cpu())
    if kind == "largest":
        return   # (logits without bounds)
    # logits below 2^5 whatever the keys' sizes
    top = float(rk.float().abs().max())
    cache, L = given(k, v, 4, 3, scale=0.5 / top)
    q = rand(gen(7), 1, 4, d)
    o, lse = spk.sparsek_cache4_attn(cache, L, q)
    torch.cuda.synchronize()
    ro, rl, _, ob = ref.cache_attn(cache, [130], q)
    assert ((ref.f64(o) - ro).abs() <= ob).all() and ((lse.cpu().double() - rl).abs() <= 2e-4).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("where", ["key", "value"])
@pytest.mark.parametrize("e", [10, 20, 27, 30, 33, 35, 36, 37, 38, 39, 100])
def test_what_a_query_does_not_weigh_does_not_move_it(where, e, d):
    """A key of 2^e in a channel where the query is 0, or a value of 2^e whose weight is 0: the others of its block keep all their bits."""
    require_gpu()
    say("cache4, an outlier beside ordinary", where, e, d)
    g = gen(14)
    k, v, q = rand(g, 1, 1, 64, d), rand(g, 1, 1, 64, d), rand(g, 1, 2, d)
    q[..., 40] = 0.0
    if where == "key":
        k[0, 0, 9, 40] = 2.0 ** e
    else:
        v[0, 0, 9, 40] = 2.0 ** e
        k[0, 0, 9] = (-1e4 * q[0, 0].float().sign()).bfloat16()
        q[0, 1] = q[0, 0]
    cache, L = given(k, v, 2, 3)
    o, lse = spk.sparsek_cache4_attn(cache, L, q)
    torch.cuda.synchronize()
    ro, rl, _, ob = ref.cache_attn(cache, [64], q)
    assert ((ref.f64(o) - ro).abs() <= ob).all() and ((lse.cpu().double() - rl).abs() <= 2e-4).all()
    assert ro.abs().max() < 10


ROWS = [[1], [63, 64, 65, 0], [700, 128, 1, 129, 513], [2000]]


@pytest.mark.parametrize("H,Hkv,d", [(1, 1, 64), (3, 1, 128), (8, 2, 128), (32, 2, 64), (25, 1, 128)])
@pytest.mark.parametrize("lens", ROWS)
def test_attention_of_a_single_token(H, Hkv, d, lens):
    require_gpu()
    say("cache4 attention", H, Hkv, d, lens)
    cache, L, _, _ = filled(21, lens, H, Hkv, d)
    cache.kt[:, :, 63], cache.vt[:, :, :, 63] = float("nan"), float("inf")   # behind the last token: anything
    q = rand(gen(22), len(lens), H, d)
    before = torch.rand(cache.mass.shape, generator=gen(23)).cuda()
    cache.mass.copy_(before)
    o, lse = spk.sparsek_cache4_attn(cache, L, q, accumulate=True)
    torch.cuda.synchronize()
    ro, rl, rm, ob = ref.cache_attn(cache, lens, q)
    assert ((ref.f64(o) - ro).abs() <= ob).all(), float(((ref.f64(o) - ro).abs() / ob).max())
    empty = torch.tensor([n == 0 for n in lens])
    assert (o[empty] == 0).all() and (lse[empty] == float("-inf")).all()
    assert ((lse.cpu().double() - rl)[~empty].abs() <= 2e-4).all()           # logits to 60: 128 products of 2^-24 each, twice
    want = ref.f64(before) + rm
    assert ((ref.f64(cache.mass) - want).abs() <= 2 ** -12 * rm + 2 ** -23 * want).all()
    o2, lse2 = spk.sparsek_cache4_attn(cache, L, q)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("H,Hkv,d,top", [(4, 4, 64, 1), (8, 2, 128, 5), (20, 1, 128, 7)])
def test_selected_blocks(H, Hkv, d, top):
    require_gpu()
    say("cache4 selection", H, Hkv, d, top)
    lens = [900, 64, 640, 641, 1, 0, 330]
    cache, L, _, _ = filled(31, lens, H, Hkv, d)
    B = len(lens)
    q = rand(gen(32), B, H, d)
    idx = spk.sparsek_cache4_select(cache, L, q, top)
    torch.cuda.synchronize()
    p8, _ = block_ref.codes_i8(ref.f64(q).view(B, Hkv, H // Hkv, d).sum(2).float())
    for b in range(B):
        for g in range(Hkv):
            nb = max(lens[b] - 1, 0) // 64
            pages = cache.table[b, g, :nb].cpu().long()
            score = (cache.km.cpu()[pages].double() @ p8[b, g].double()).float() * cache.kms.cpu()[pages]
            assert idx[b, g].tolist() == block_ref.top_of(score, [True] * nb, top), (b, g)
    other = torch.randint(-4, 20, idx.shape, generator=gen(33), dtype=torch.int32).cuda()
    other[0, :, top // 2:] = 3
    other[2, :, 0] = 2 ** 31 - 1
    for x in (idx, other, torch.full_like(idx, -1), idx[..., :0]):
        cache.mass.zero_()
        o, lse = spk.sparsek_cache4_attn(cache, L, q, x.contiguous(), accumulate=True)
        torch.cuda.synchronize()
        ro, rl, rm, ob = ref.cache_attn(cache, lens, q, x.cpu())
        assert ((ref.f64(o) - ro).abs() <= ob).all()
        assert ((ref.f64(cache.mass) - rm).abs() <= 2 ** -12 * rm).all()
        some = torch.tensor([n > 0 for n in lens])
        assert ((lse.cpu().double() - rl)[some].abs() <= 2e-4).all()


def test_pages_outside_the_pool_are_attended_by_nobody():
    require_gpu()
    say("cache4 attention, bad pages")
    cache, L, _, _ = filled(41, [500, 300], 4, 2, 64)
    cache.table[0, 0, 2], cache.table[0, 1, 0], cache.table[1, 1] = -1, cache.cfg.pages, -7
    q = rand(gen(42), 2, 4, 64)
    o, lse = spk.sparsek_cache4_attn(cache, L, q, accumulate=True)
    torch.cuda.synchronize()
    ro, rl, rm, ob = ref.cache_attn(cache, [500, 300], q)
    assert ((ref.f64(o) - ro).abs() <= ob).all()
    assert ((ref.f64(cache.mass) - rm).abs() <= 2 ** -12 * rm).all()


@pytest.mark.parametrize("cap,lens,budget,sink,recent", [(5, [320 + 17, 5, 256, 0], 3, 1, 1), (40, [2560, 2000, 64 * 40 + 63, 64 * 12], 12, 2, 3)])
def test_eviction(cap, lens, budget, sink, recent):
    require_gpu()
    say("cache4 eviction", cap, lens, budget, sink, recent)
    cache = shuffled(spk.Cache4.empty(len(lens), 3, 3, 64, cap), 51)
    mass = torch.exp(2 * torch.randn(len(lens), 3, cap, generator=gen(52)))
    mass[:, 1] = 1.0
    cache.mass.copy_(mass)
    L = ints(lens)
    out = spk.sparsek_cache4_evict(cache, L, budget, sink, recent)
    torch.cuda.synchronize()
    for got, want in zip((out["table"], out["mass"], out["lens"]), block_ref.evict(cache.table, cache.mass, L, budget, sink, recent)):
        assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("begin,n", [(0, 1), (63, 2), (64, 64), (1, 200), (130, 500), (511, 1), (700, 40)])
@pytest.mark.parametrize("d", [64, 128])
def test_ranges_that_are_read(begin, n, d):
    """From the middle of a block to the middle of another, and past the end; what was not asked for is not written."""
    require_gpu()
    say("cache4 read", begin, n, d)
    lens = [600, 64, 0, 511]
    cache, L, k, v = filled(55, lens, 2, 2, d)
    all_k, all_v = spk.sparsek_cache4_read(cache, L, 0, 800)
    room = torch.full((2, 4 * 2 * n * d + 256), 5.0, dtype=torch.bfloat16, device="cuda")
    out = tuple(x[128:-128].view(4, 2, n, d) for x in room)
    rk, rv = spk.sparsek_cache4_read(cache, L, begin, n, out=out)
    torch.cuda.synchronize()
    assert rk is out[0] and (room[:, :128] == 5).all() and (room[:, -128:] == 5).all()
    for b, m in enumerate(lens):
        assert torch.equal(ref.f64(all_k[b, :, :m]), as_held(k[b], m, -1)) and (all_k[b, :, m:] == 0).all()
    assert torch.equal(rk, all_k[:, :, begin:begin + n]) and torch.equal(rv, all_v[:, :, begin:begin + n])


@pytest.mark.parametrize("cap", [4, 40])   # one workgroup has all of it, or several
@pytest.mark.parametrize("where", ["key", "value", "last token's key", "last token's value"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_values_that_are_not_finite_reach_who_attends_them(bad, where, cap):
    require_gpu()
    say("cache4, not finite:", bad, where, cap)
    B, H, Hkv, d, n = 2, 4, 2, 64, 220
    g = gen(5)
    k, v, q = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d), rand(g, B, H, d)
    q[1, 2:, 9] = q[1, 2:, 9].abs() + 1
    last = where.startswith("last")
    without = ints([0, 2]).expand(B, Hkv, 2).contiguous()

    def run(k, v):
        cache, L = given(k, v, H, cap)
        return spk.sparsek_cache4_attn(cache, L, q, accumulate=True) + spk.sparsek_cache4_attn(cache, L, q, without) + spk.sparsek_cache4_read(cache, L, 0, n)

    clean = run(k, v)
    (k if "key" in where else v)[1, 1, n - 1 if last else 100, 9] = bad
    got = run(k, v)
    torch.cuda.synchronize()
    for x, (a, want) in enumerate(zip(got[:4], clean)):
        mine = a[1, 2:]
        if where == "last token's key" and bad == float("-inf"):   # (a weight of 0)
            assert torch.isfinite(mine).all()
        elif last and "value" in where and x in (0, 2):
            assert not torch.isfinite(mine[:, 9]).any(), x
        elif x == 0 or last and x == 2:
            assert torch.isnan(mine).all(), x
        elif x == 2:   # (without the second block)
            assert torch.equal(mine, want[1, 2:])
        assert torch.equal(a[0], want[0]) and torch.equal(a[1, :2], want[1, :2]), x
    for a, want, mine in zip(got[4:], clean[4:], ("key", "value")):   # read: all of the page, or the one value of the last token
        want = want.clone()
        if mine in where:
            if last:
                want[1, 1, n - 1, 9] = bad
            else:
                want[1, 1, 64:128] = float("nan")
        assert same(a, want)


@pytest.mark.parametrize("cap,n", [(4, 220), (40, 220), (40, 128), (4, 30)])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_a_query_that_is_not_finite_gets_nan(value, cap, n):
    require_gpu()
    say("cache4 attention, a query of", value, cap, n)
    B, H, Hkv, d = 3, 4, 2, 64
    g = gen(35)
    k, v, q = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d), rand(g, B, H, d)
    k[..., 7] = 4.0     # (no code of 0 in the column)
    cache, L = given(k, v, H, cap)
    L[2] = 0
    runs = []
    for x in (0.5, value):
        q[1:, 1, 7] = x
        runs.append(spk.sparsek_cache4_attn(cache, L, q))
    torch.cuda.synchronize()
    (o, lse), (o1, lse1) = runs
    assert torch.isnan(o1[1, 1]).all() and torch.isnan(lse1[1, 1])
    assert (o1[2] == 0).all() and (lse1[2] == float("-inf")).all()
    o1[1, 1], lse1[1, 1] = o[1, 1], lse[1, 1]
    assert torch.equal(o, o1) and torch.equal(lse, lse1)


@pytest.mark.parametrize("cap,n", [(4, 220), (40, 220), (40, 128)])
@pytest.mark.parametrize("e", [8, 20, 24, 27, 60])
def test_logits_of_all_sizes(e, cap, n):
    """Logits up to 2^e: the weights are the largest ones' alone, which share a code."""
    require_gpu()
    say("cache4 attention, logits of 2^%d" % e, cap, n)
    g = gen(55)
    c = torch.tensor([0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])[torch.randint(0, 7, (n,), generator=g)]
    k = c.view(1, 1, n, 1).expand(1, 1, n, 64).bfloat16().contiguous().cuda()   # (a token's values are all one code)
    v, q = rand(g, 1, 1, n, 64), torch.ones(1, 2, 64).bfloat16().cuda()
    cache, L = given(k, v, 2, cap, scale=0.7 * 2.0 ** e / (64 * 6))
    o, lse = spk.sparsek_cache4_attn(cache, L, q)
    torch.cuda.synchronize()
    ro, rl, rm, ob = ref.cache_attn(cache, [n], q)
    if e >= 20:
        assert ((ref.f64(o) - ro).abs() <= ob + 2 ** -11 * ro.abs()).all()
    else:
        assert ((ref.f64(o) - ro).abs() <= ob + 2 ** -22 * 2 ** e * ro.abs().amax()).all()
    assert ((lse.cpu().double() - rl).abs() <= 2 ** -21 * rl.abs() + 2 ** -20).all()


def test_the_longest_table():
    """8192 blocks of a row that share 64 pages, over all and over a selection longer than a workgroup's share with repeated places."""
    require_gpu()
    say("cache4 of 8192 blocks")
    B, H, d, cap = 1, 2, 64, 8192
    cache = spk.Cache4.empty(B, H, 1, d, cap, pages=64)
    g = gen(81)
    lens = torch.zeros(B, dtype=torch.int32).cuda()
    spk.sparsek_cache4_append(cache, lens, rand(g, B, 1, 64 * 64, d), rand(g, B, 1, 64 * 64, d))
    cache.table.copy_(torch.randint(0, 64, cache.table.shape, generator=g, dtype=torch.int32))
    cache.kt.copy_(rand(g, *cache.kt.shape))
    cache.vt.copy_(rand(g, *cache.vt.shape))
    L = cap * 64 + 63
    lens = ints([L])
    q = rand(g, B, H, d)
    many = torch.randint(-5, 5200, (B, 1, 300), generator=g, dtype=torch.int32)
    many[:, :, 200:] = many[:, :, :100]
    pages = [ref.dequantised(cache, p) for p in range(64)]
    at = cache.table[0, 0].cpu().long()
    for x in (None, many):
        places = list(range(cap)) if x is None else sorted({int(y) for y in x[0, 0] if 0 <= int(y) < cap})
        K = torch.cat([pages[at[j]][0] for j in places] + [ref.f64(cache.kt[0, 0, :63])])
        V = torch.cat([pages[at[j]][1] for j in places] + [ref.f64(cache.vt[0, 0, :, :63]).T])
        o, lse = spk.sparsek_cache4_attn(cache, lens, q, None if x is None else x.cuda())
        torch.cuda.synchronize()
        for h in range(H):
            s = K @ ref.f64(q[0, h]) * cache.cfg.softmax_scale
            p = torch.softmax(s, 0)
            want = p @ V
            assert ((ref.f64(o[0, h]) - want).abs() <= 2 ** -8 * want.abs() + (2 ** -11 + 2 ** -14) * (p @ V.abs())).all()
            assert abs(float(lse[0, h]) - float(torch.logsumexp(s, 0))) <= 2e-4


def test_calls_on_streams_of_their_own():
    require_gpu()
    say("cache4 steps on two streams")
    made = [filled(90 + x, [700 + 60 * x, 90], 8, 2, 128, cap=14) for x in range(2)]
    q = [rand(gen(95 + x), 2, 8, 128) for x in range(2)]
    torch.cuda.synchronize()
    want = [spk.sparsek_cache4_attn(c, L, y) + spk.sparsek_cache4_read(c, L, 3, 300) for (c, L, _, _), y in zip(made, q)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for x in range(2):
            with torch.cuda.stream(streams[x]):
                got[x].append(spk.sparsek_cache4_attn(made[x][0], made[x][1], q[x]) + spk.sparsek_cache4_read(made[x][0], made[x][1], 3, 300))
    torch.cuda.synchronize()
    for x in range(2):
        for run in got[x]:
            assert all(torch.equal(a, b) for a, b in zip(run, want[x]))


def test_a_conversation():
    """Projections' outputs normed and turned by their positions, prefill over selected blocks, its keys, values and masses into the cache, then
    tokens one by one with eviction: every step against the definition on what the cache then holds."""
    require_gpu()
    say("a conversation over the cache in 4 bits")
    B, H, Hkv, d, n, top, cap, budget = 2, 4, 2, 64, 300, 3, 8, 4
    g = gen(61)
    more = 90
    x = rand(g, B, n + more, (H + 2 * Hkv) * d)
    q, k = x[..., :H * d].unflatten(-1, (H, d)), x[..., H * d:(H + Hkv) * d].unflatten(-1, (Hkv, d))
    v = x[..., (H + Hkv) * d:].unflatten(-1, (Hkv, d)).transpose(1, 2).contiguous()
    pos = torch.arange(n + more, dtype=torch.int32).expand(1, B, n + more).contiguous().cuda()
    freq = (10000.0 ** (-torch.arange(32) / 32.0)).float().cuda()
    w = (1 + 0.2 * torch.randn(2, d, generator=g)).cuda()
    args = dict(norm=True, qw=w[0], kw=w[1])
    qo, ko = spk.sparsek_rope_fwd(q[:, :n], k[:, :n], pos[:, :, :n].contiguous(), freq, **args)
    idx = spk.sparsek_block_select(qo, ko, top)
    o, lse, mass = spk.sparsek_block_attn_fwd(qo, ko, v[:, :, :n].contiguous(), idx, d ** -0.5, mass=True)
    cache = spk.Cache4.empty(B, H, Hkv, d, cap)
    lens = torch.zeros(B, dtype=torch.int32).cuda()
    spk.sparsek_cache4_append(cache, lens, ko, v[:, :, :n].contiguous())
    lens = lens + n
    cache.mass[:, :, :mass.shape[2]] = mass
    for t in range(n, n + more):
        if int(lens[0]) // 64 > budget:
            out = spk.sparsek_cache4_evict(cache, lens, budget, 1, 2)
            cache.adopt(out["table"], out["mass"])
            lens = out["lens"]
        qt, kt = spk.sparsek_rope_fwd(q[:, t:t + 1], k[:, t:t + 1], pos[:, :, t:t + 1].contiguous(), freq, **args)
        spk.sparsek_cache4_append(cache, lens, kt, v[:, :, t:t + 1].contiguous())
        lens = lens + 1
        qt = qt[:, :, 0]
        sel = spk.sparsek_cache4_select(cache, lens, qt, top) if t % 2 else None
        o, lse = spk.sparsek_cache4_attn(cache, lens, qt, sel, accumulate=True)
        if t % 23 == 0 or t < n + 3:
            torch.cuda.synchronize()
            for y, z, wt in ((qt, q, w[0]), (kt[:, :, 0], k, w[1])):
                want, bound = rope_ref.fwd(z[:, t:t + 1], pos[:, :, t:t + 1], freq, None, False, True, wt, 1e-6)
                assert ((ref.f64(y) - want[:, :, 0]).abs() <= bound[:, :, 0]).all()
            ro, rl, rm, ob = ref.cache_attn(cache, lens.tolist(), qt, None if sel is None else sel.cpu())
            assert ((ref.f64(o) - ro).abs() <= ob).all(), t
    assert (cache.mass >= 0).all() and torch.isfinite(cache.mass).all()


def test_decode_step_replays_as_a_graph():
    """One step captured (positions and lengths move on inside the graph), replayed over the end of a block, against eager steps; and two
    graphs with workspaces of their own replayed in turn."""
    require_gpu()
    say("cache4 step as a graph")
    B, H, Hkv, d = 2, 8, 2, 128
    lens0 = [250, 190]
    freq = (10000.0 ** (-torch.arange(64) / 64.0)).float().cuda()

    def fresh():
        return filled(71, lens0, H, Hkv, d, cap=6)[:2]

    def step(cache, lens, q, k, v):
        qo, ko = spk.sparsek_rope_fwd(q, k, lens.view(1, B, 1), freq, norm=True)
        spk.sparsek_cache4_append(cache, lens, ko, v)
        lens.add_(1)
        qo = qo[:, :, 0]
        idx = spk.sparsek_cache4_select(cache, lens, qo, 2)
        return spk.sparsek_cache4_attn(cache, lens, qo, idx, accumulate=True) + spk.sparsek_cache4_attn(cache, lens, qo) + spk.sparsek_cache4_read(cache, lens, 180, 80)

    g = gen(72)
    new = [(rand(g, B, 1, H, d), rand(g, B, 1, Hkv, d), rand(g, B, Hkv, 1, d)) for _ in range(10)]
    ec, el = fresh()
    eager = []
    for x in new:
        eager.append([t.clone() for t in step(ec, el, *x)])
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        cache, lens = fresh()
        q, k, v = (t.clone() for t in new[0])
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            wc, wl = fresh()
            step(wc, wl, q, k, v)
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(cache, lens, q, k, v)
        graphs.append((graph, cache, lens, (q, k, v), out))
    for i, x in enumerate(new):
        for graph, cache, lens, args, out in graphs:
            for dst, src in zip(args, x):
                dst.copy_(src)
            graph.replay()
        torch.cuda.synchronize()
        for graph, cache, lens, args, out in graphs:
            for a, b in zip(out, eager[i]):
                assert torch.equal(a, b), i
    for _, cache, lens, _, _ in graphs:
        assert torch.equal(cache.mass, ec.mass) and torch.equal(lens, el)
        assert torch.equal(cache.k4, ec.k4) and torch.equal(cache.ve, ec.ve) and torch.equal(cache.kt, ec.kt)


def test_pages_beyond_32_bits():
    """A pool of more than 2^32 bytes: its last pages hold what its first ones would."""
    require_gpu()
    say("cache4, pages beyond 2^32 bytes")
    B, H, Hkv, d, cap, n = 1, 4, 2, 128, 8, 400
    g = gen(101)
    k, v, q = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d), rand(g, B, H, d)
    runs = []
    for pages in (16, 2 ** 20 + 40):
        cache = spk.Cache4.empty(B, H, Hkv, d, cap, pages=pages)
        cache.table.copy_(torch.arange(pages - 16, pages, dtype=torch.int32).view(B, Hkv, cap))
        L = ints([n])
        spk.sparsek_cache4_append(cache, torch.zeros_like(L), k, v)
        idx = spk.sparsek_cache4_select(cache, L, q, 3)
        runs.append(spk.sparsek_cache4_attn(cache, L, q, accumulate=True) + spk.sparsek_cache4_attn(cache, L, q, idx) + spk.sparsek_cache4_read(cache, L, 0, n))
        runs[-1] += (idx, cache.mass.clone(), cache.ke[-16:].clone())
        torch.cuda.synchronize()
        assert pages == 16 or (cache.k4[:64] == 0).all() and cache.k4.numel() > 2 ** 32
        del cache
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv,B,n", [(40, 2, 2, 700), (16, 16, 20, 2400), (8, 8, 40, 2400), (8, 8, 1, 1900), (4, 4, 1, 9000), (6, 2, 3, 20000)])
def test_one_workgroup_or_many(H, Hkv, B, n, d):
    """Every way in which a sequence is shared out: more heads than a product has columns, one workgroup for few blocks, for up to 40 of them where
    there are many sequences, few parts and many parts of a sequence; all with the masses of all blocks."""
    require_gpu()
    say("cache4, shared out", H, Hkv, B, n, d)
    g = gen(111)
    base = rand(g, 1, Hkv, n, d), rand(g, 1, Hkv, n, d)
    cache = spk.Cache4.empty(B, H, Hkv, d, n // 64 + 1, pages=Hkv * (n // 64 + 1))
    cache.table.copy_(torch.arange(Hkv * (n // 64 + 1), dtype=torch.int32).view(1, Hkv, -1).expand_as(cache.table))   # (all sequences have the same pages)
    one = spk.Cache4(cache.k4, cache.v4, cache.ke, cache.ve, cache.ks, cache.vs, cache.km, cache.kms, cache.kt[:1].clone(), cache.vt[:1].clone(),
                     cache.table[:1].clone(), cache.mass[:1].clone(), H, d ** -0.5)
    spk.sparsek_cache4_append(one, ints([0]), *base)
    cache.kt.copy_(one.kt.expand_as(cache.kt))
    cache.vt.copy_(one.vt.expand_as(cache.vt))
    whole = n // 64 * 64
    lens = [n if b == 0 else whole - 64 * (b % (n // 64)) for b in range(B)]   # (others end with a block, so that the unfinished one is nobody's)
    q = rand(g, B, H, d)
    o, lse = spk.sparsek_cache4_attn(cache, ints(lens), q, accumulate=True)
    torch.cuda.synchronize()
    for b in sorted({0, B // 2, B - 1}):
        cut = type("C", (), dict(B=1, H=H, Hkv=Hkv, d=d, cap=cache.cap, cfg=cache.cfg, k4=cache.k4, v4=cache.v4, ke=cache.ke, ve=cache.ve, ks=cache.ks,
                                 vs=cache.vs, kt=cache.kt[b:b + 1], vt=cache.vt[b:b + 1], table=cache.table[b:b + 1]))
        ro, rl, rm, ob = ref.cache_attn(cut, lens[b:b + 1], q[b:b + 1])
        assert ((ref.f64(o[b:b + 1]) - ro).abs() <= ob).all()
        assert ((lse[b:b + 1].cpu().double() - rl).abs() <= 2e-4).all()
        assert ((ref.f64(cache.mass[b:b + 1]) - rm).abs() <= 2 ** -12 * rm).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(4, 2), (40, 2)])
def test_wide_pages_among_others(H, Hkv, d):
    """Pages whose scales lie far apart in keys, in values or in both, beside ordinary ones, ones with a value that is not finite, and ones outside the
    pool: over all tokens and over chosen blocks, with the masses."""
    require_gpu()
    say("cache4, wide pages among others", H, Hkv, d)
    B, n = 2, 700
    g = gen(121)
    k, v, q = rand(g, B, Hkv, n, d), rand(g, B, Hkv, n, d), rand(g, B, H, d)
    far, off = (torch.exp2(torch.randint(-60, 1, s, generator=g).float()).cuda().bfloat16() for s in ((B, Hkv, n, 1), (B, Hkv, 1, d)))   # (32 share a scale)
    block = torch.arange(n).cuda() // 64
    k = torch.where((block % 3 == 1).view(1, 1, n, 1), k * far, k)
    v = torch.where((block % 4 >= 2).view(1, 1, n, 1), v * off, v)
    cap = n // 64 + 1
    cache, L = given(k, v, H, cap)
    cache.table[1, 0, 4] = -1
    wide = (cache.ks.view(torch.int32) & 0x7FFFFF) != 0, (cache.vs.view(torch.int32) & 0x7FFFFF) != 0
    assert all(x.any() and not x.all() for x in wide)
    idx = ints([1, 2, 4, 7]).expand(B, Hkv, 4).contiguous()
    for x in (None, idx):
        cache.mass.zero_()
        o, lse = spk.sparsek_cache4_attn(cache, L, q, x, accumulate=True)
        torch.cuda.synchronize()
        ro, rl, rm, ob = ref.cache_attn(cache, [n] * B, q, None if x is None else x.cpu())
        assert ((ref.f64(o) - ro).abs() <= ob).all(), float(((ref.f64(o) - ro).abs() / ob).max())
        assert ((lse.cpu().double() - rl).abs() <= 2e-4).all()
        assert ((ref.f64(cache.mass) - rm).abs() <= 2 ** -12 * rm).all()
    # a key that is not finite in a block whose values are wide, and a value in one whose keys are
    for x, b, at in ((k, 0, 64 * 3 + 5), (v, 1, 64 * 1 + 9)):
        x[b, 1, at, 11] = float("nan")
    cache, L = given(k, v, H, cap)
    o, lse = spk.sparsek_cache4_attn(cache, L, q)
    torch.cuda.synchronize()
    ro, rl, _, ob = ref.cache_attn(cache, [n] * B, q)
    bad = torch.zeros(B, H, dtype=torch.bool)
    bad[0, H // 2:] = bad[1, H // 2:] = True
    assert torch.isnan(o[bad.cuda()]).all() and torch.isnan(lse[0, H // 2:]).all() and torch.isfinite(lse[1]).all()
    assert ((ref.f64(o) - ro).abs() <= ob)[~bad].all()


def close(cache, lens, q, o, lse):
    """Bounds of the attention with weights as two bf16 numbers: 2^-8 of what is rounded to bf16, 2^-16 of a weight (each of the two roundings 2^-8), and 2^-14
    for sums in fp32 and exponentials (exponents up to 93 of two, of products rounded twice to fp32: 93 * 2^-23 * ln 2 = 2^-17)."""
    torch.cuda.synchronize()
    B, H, d = q.shape
    G = H // cache.Hkv
    for b in range(B):
        for h in range(H):
            K, V, _, _, _ = ref.row_tokens(cache, lens, b, h // G)
            s = K @ ref.f64(q[b, h]) * cache.cfg.softmax_scale
            p = torch.softmax(s, 0)
            want, bound = p @ V, 2 ** -8 * (p @ V).abs() + (2 ** -16 + 2 ** -14) * (p @ V.abs())
            e = (ref.f64(o[b, h]) - want).abs()
            assert (e <= bound).all(), float((e / bound).max())
            assert abs(float(lse[b, h]) - float(torch.logsumexp(s, 0))) <= 2e-4


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("at,n", [(9, 64), (9, 200), (70, 200), (194, 200), (9, 2000), (1500, 2000)])
@pytest.mark.parametrize("key,e", [(-16, 20), (-16, 27), (-16, 40), (-24, 30), (-24, 36), (-32, 45), (-32, 60), (-64, 100)])
def test_large_values_of_small_weights(key, e, at, n, d):
    """A value of 2^e whose weight is exp(key) of the others', in their block, in another and in the unfinished one: what it adds is its product."""
    require_gpu()
    say("cache4, large values of small weights", key, e, at, n, d)
    g = gen(131)
    k, v, q = torch.zeros(1, 1, n, d).bfloat16().cuda(), rand(g, 1, 1, n, d), torch.zeros(1, 2, d).bfloat16().cuda()
    q[:, 0, 0], q[:, 1, 0] = 1.0, 0.5
    k[0, 0, at, 0] = key
    v[0, 0, at, ::3] = 2.0 ** e
    cache, L = given(k, v, 2, 40, scale=1.0)
    close(cache, [n], q, *spk.sparsek_cache4_attn(cache, L, q))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,n", [(3, 150), (40, 150), (40, 128)])
@pytest.mark.parametrize("e", [60, 105, 112, 114, 118])
def test_values_of_all_sizes(e, cap, n, d):
    """Outputs of up to 2^e are finite, whether a block is whole or not.  (150 of them, four standard deviations each, sum up to less than 2^(e+10).)"""
    require_gpu()
    say("cache4, values of 2^%d" % e, cap, n, d)
    g = gen(141)
    k, v, q = rand(g, 1, 2, n, d), rand(g, 1, 2, n, d) * 2.0 ** e, rand(g, 1, 4, d)
    cache, L = given(k, v, 4, cap)
    close(cache, [n], q, *spk.sparsek_cache4_attn(cache, L, q))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("e", [10, 17, 20, 24, 30, 36, 60])
def test_small_channels_of_queries_and_large_ones_of_keys(e, d):
    """A query's channel of 2^-e meets keys of 2^e there: logits are as with 1 and 1."""
    require_gpu()
    say("cache4, small channels of queries", e, d)
    g = gen(151)
    n = 200
    k, v, q = rand(g, 1, 1, n, d), rand(g, 1, 1, n, d), rand(g, 1, 2, d)
    k[..., 3] = torch.tensor([-4.0, -2.0, 0.5, 1.0, 3.0, 6.0]).bfloat16().cuda()[torch.randint(0, 6, (n,), generator=g).cuda()] * 2.0 ** e
    q[..., 3] = torch.tensor([3.0, -5.0]).cuda() * 2.0 ** -e
    cache, L = given(k, v, 2, 4)
    close(cache, [n], q, *spk.sparsek_cache4_attn(cache, L, q))


@pytest.mark.parametrize("d,n,begin", [(64, 33001, 37), (128, 17001, 130)])
def test_long_ranges_that_are_read(d, n, begin):
    """Outputs of more than 100 MB, which go past the caches: every stretch has the bits that it has in a short read, over lengths inside and outside the range,
    a page with a value that is not finite and pages outside the pool; what was not asked for is not written."""
    require_gpu()
    say("cache4 long read", d, n, begin)
    lens, Hkv = [begin + n + 200, 9017, 0], 4
    assert 4 * len(lens) * Hkv * n * d > 100e6
    cap = (begin + n) // 64 + 5
    cache, g = shuffled(spk.Cache4.empty(len(lens), Hkv, Hkv, d, cap), 161), gen(162)
    k, v = (torch.randn(Hkv, 4000, d, generator=g).bfloat16().cuda()[:, torch.arange(max(lens), device="cuda") % 4000].expand(len(lens), -1, -1, -1).contiguous()
            for _ in range(2))
    k[0, 1, 700, 3], v[1, 2, 5000, 9] = float("nan"), float("inf")
    L = ints(lens)
    spk.sparsek_cache4_append(cache, torch.zeros_like(L), k, v, counts=L)
    cache.table[0, 3, 40], cache.table[1, 0, 30] = -1, cache.cfg.pages
    room = torch.full((2, len(lens) * Hkv * n * d + 256), 5.0, dtype=torch.bfloat16, device="cuda")
    out = tuple(x[128:-128].view(len(lens), Hkv, n, d) for x in room)
    rk, rv = spk.sparsek_cache4_read(cache, L, begin, n, out=out)
    torch.cuda.synchronize()
    assert (room[:, :128] == 5).all() and (room[:, -128:] == 5).all()
    for a in range(0, n, 4001):
        c = min(4001, n - a)
        for got, want in zip((rk, rv), spk.sparsek_cache4_read(cache, L, begin + a, c)):
            assert torch.equal(got[:, :, a:a + c].contiguous().view(torch.int16), want.view(torch.int16)), a
    assert rk[0, 1].isnan().any() and rv[1, 2].isnan().any() and not rk[1].isnan().any()
    assert (rk[1, :, 9017 - begin:] == 0).all() and (rv[2] == 0).all() and (rk[0, 3, 40 * 64 - begin:41 * 64 - begin] == 0).all()
    clean = slice(10 * 64, 20 * 64)
    for got, given_, dim in ((rk, k, -1), (rv, v, -2)):
        want = ref.rounded(given_[0, 0, clean].unflatten(0, (-1, 64)), dim).flatten(0, 1)
        assert torch.equal(ref.f64(got[0, 0, 10 * 64 - begin:20 * 64 - begin]), want)


def test_reading_more_than_2_31_values():
    require_gpu()
    say("cache4 read of more than 2^31 values")
    B, Hkv, d, cap, n = 8, 4, 128, 8192, 530000
    assert B * Hkv * n * d > 2 ** 31
    cache, g = spk.Cache4.empty(B, Hkv, Hkv, d, cap, pages=64 * B * Hkv), gen(171)
    spk.sparsek_cache4_append(cache, torch.zeros(B, dtype=torch.int32).cuda(), rand(g, B, Hkv, 4096, d), rand(g, B, Hkv, 4096, d))
    cache.table.copy_(torch.randint(0, 64 * B * Hkv, cache.table.shape, generator=g, dtype=torch.int32))
    cache.kt.copy_(rand(g, *cache.kt.shape))
    cache.vt.copy_(rand(g, *cache.vt.shape))
    lens = ints([cap * 64 + 63, 500, 100000, 0, 1, 300000, 64 * 8000, cap * 64 + 63])
    rk, rv = spk.sparsek_cache4_read(cache, lens, 0, n)
    for a in (0, 99900, 299900, cap * 64 - 100):
        for got, want in zip((rk, rv), spk.sparsek_cache4_read(cache, lens, a, 300)):
            assert torch.equal(got[:, :, a:a + 300], want), a
    torch.cuda.synchronize()
    assert (rk[7, 3, cap * 64 + 63:] == 0).all() and (rk[7, 3, :cap * 64 + 63].abs().amax(-1) > 0).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [128, 150, 2000])
@pytest.mark.parametrize("eq,ek", [(0, 100), (0, 123), (60, 60), (100, 20), (0, -95), (-60, -30), (-100, 100), (-20, 120)])
def test_queries_and_keys_of_all_sizes(eq, ek, n, d):
    """Queries of 2^eq and keys of 2^ek whose scale makes ordinary logits of them: products beyond fp32's range are no logits beyond it."""
    require_gpu()
    say("cache4, queries and keys of all sizes", eq, ek, n, d)
    g = gen(181)
    k, v, q = rand(g, 1, 2, n, d) * 2.0 ** ek, rand(g, 1, 2, n, d), rand(g, 1, 4, d) * 2.0 ** eq
    cache, L = given(k, v, 4, 40, scale=d ** -0.5 * 2.0 ** (-eq - ek))
    close(cache, [n], q, *spk.sparsek_cache4_attn(cache, L, q))
